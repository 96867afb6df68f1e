// The gated block's forward pass in one kernel, for input and output widths up
// to 64: a coordinate network's first and last layers.
#pragma once

#include <algorithm>

#include "net_common.hpp"
#include "net_plans.hpp"

namespace fd {
namespace net {

constexpr int64_t NARROW_ROWS = 128;  // of a workgroup
// Parts of F until every CU has a workgroup, two steps each at least.
inline int narrow_parts(int64_t N, int64_t F) {
  const int64_t want = 256 / std::max<int64_t>(1, ceil_div(N, NARROW_ROWS));
  return int(std::max<int64_t>(1, std::min({want, ceil_div(F, int64_t(64)), int64_t(32)})));
}

struct NarrowArgs {
  fd_gated_block b;
  const void* R;
  int64_t ldr;
  void* Y;
  int64_t ldy;
  char* saved;  // G and U by blocks, or NULL
  int64_t Fp;
  // parts of F, each with its own workgroups; where more than one, part s of Y
  // is at part + s N ldp in float32, without bd and R
  int parts;
  float* part;
  int64_t ldp;
};

// planes: of H, between its two products.
void run_narrow(const NarrowArgs& p, int planes, hipStream_t stream);

}  // namespace net
}  // namespace fd
