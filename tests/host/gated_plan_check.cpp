// CPU driver of the gated block's plans (net_plans.hpp), built by
// tests/test_host_gated_plans.py.
//
//   list    for each line "type N D F O" of the input (type: f32, bf16, bf16x2, where the last holds
//           H, dG and dU in two planes), the kernels that its passes take, a line each
//   reach   the kernels that sizes drawn over the operators' range take, each with the
//           cheapest size that takes it
//
// A kernel is named by type, product, tile and whether its contraction is split.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <map>
#include <random>
#include <set>
#include <string>

#include "net_plans.hpp"

using namespace fd;
using namespace fd::net;

struct Size {
  int64_t N, D, F, O;
};

static std::string kernel(const char* type, const char* product, int config, const Shape& s) {
  static const char* tiles[CONFIGS] = {"big", "mid", "small"};
  return std::string(type) + " " + product + " " + tiles[config] + (s.splits > 1 ? " split" : " whole");
}

static std::set<std::string> kernels(const char* type, const Size& z) {
  const bool f32 = std::strcmp(type, "f32") == 0, fine = std::strcmp(type, "bf16x2") == 0;
  std::set<std::string> out;
  const Way way = forward_way(z.N, z.D, z.O, f32, false);
  if (way == FEW_ROWS) out.insert(std::string(type) + " few rows");
  // with G and U kept, the pass of few rows goes on by the other two
  if (forward_way(z.N, z.D, z.O, f32, true) == NARROW_WAY) {
    out.insert(std::string(type) + " narrow");
  } else {
    const GatedPlan p = plan_gated(z.N, z.D, z.F, z.O, f32, fine, 0);
    out.insert(kernel(type, "gate", p.gate_config, p.gate));
    out.insert(kernel(type, "y", p.config, p.out[0]));
  }
  const GatedPlan p = plan_gated(z.N, z.D, z.F, z.O, f32, fine, 2);
  out.insert(kernel(type, "gate", p.gate_config, p.gate));  // made again
  out.insert(kernel(type, "grad", p.grad_config, p.grad));
  static const char* names[GROUP_GEMMS] = {"dx", "dw", "dwd"};
  for (int i = 0; i < GROUP_GEMMS; ++i) out.insert(kernel(type, names[i], p.config, p.out[i]));
  return out;
}

static void list() {
  char type[16];
  long long n, d, f, o;
  while (std::scanf("%15s %lld %lld %lld %lld", type, &n, &d, &f, &o) == 5)
    for (const std::string& k : kernels(type, Size{n, d, f, o})) std::printf("%s\n", k.c_str());
}

static void reach(int count) {
  std::mt19937_64 rng(1);
  auto size = [&](double lo, double hi) {
    std::uniform_real_distribution<double> u(std::log(lo), std::log(hi));
    return int64_t(std::exp(u(rng)) + 0.5);
  };
  std::map<std::string, std::pair<double, Size>> best;
  for (int i = 0; i < count; ++i) {
    const Size z{size(1, 65536), size(4, 2048), size(16, 8192), size(4, 2048)};
    const double work = double(z.N) * double(z.F) * double(2 * z.D + z.O);
    if (work > 2.7e11 * 3 || z.N * z.F > int64_t(1) << 27) continue;
    const double longest = double(z.N) * double(z.F) * double(std::max(z.D, z.O));
    const char* types[3] = {"f32", "bf16", "bf16x2"};
    for (const char* type : types) {
      // one plane above the line; two below it, or above where the caller asks
      if (std::strcmp(type, "bf16") == 0 && longest <= double(1 << 25)) continue;
      for (const std::string& k : kernels(type, z)) {
        auto it = best.find(k);
        if (it == best.end() || work < it->second.first) best[k] = {work, z};
      }
    }
  }
  for (const auto& b : best)
    std::printf("%s: %lld %lld %lld %lld\n", b.first.c_str(), (long long)b.second.second.N,
                (long long)b.second.second.D, (long long)b.second.second.F,
                (long long)b.second.second.O);
}

int main(int argc, char** argv) {
  if (argc == 2 && std::strcmp(argv[1], "list") == 0) return list(), 0;
  if (argc == 2 && std::strcmp(argv[1], "reach") == 0) return reach(30000), 0;
  std::fprintf(stderr, "usage: gated_plan_check list | reach\n");
  return 2;
}
