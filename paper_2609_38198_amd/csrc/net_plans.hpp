// Host logic of the gated block's products: which kernels a call takes, in which
// tiles, and in how many parts of their contractions.  No HIP in here, so that a CPU
// build can ask what a size takes.
#pragma once

#include <algorithm>
#include <cmath>

#include "fd_plans.hpp"

namespace fd {
namespace net {

constexpr int F_PAD = 64;       // inner widths are padded to whole k tiles
constexpr int GROUP_GEMMS = 3;  // products of a launch at most
inline int64_t f_padded(int64_t F) { return round_up(F, F_PAD); }
constexpr int k_extent(bool f32) { return f32 ? 32 : 64; }  // k of an LDS tile

// What a product does with its accumulators.
enum Epilogue {
  STORE = 0,  // C (+ bias + R) in T, or a split's float32 partial sums
  GATE = 1,   // B is [Wg; Wu]: H = act(G) U as planes, G and U kept where wanted
  GRAD = 2    // C is dH: dG, dU, H as planes from the kept G and U, column sums
};

// Tiles of C and what they cost on an MI355X (us, measured at 256 to 16384 rows
// x 512 to 2048 -> 2048 to 8192 and ragged ones): a k tile as a CU's share among as many workgroups
// as fit (operands by rows; by columns, where small tiles read LDS in twice as many
// instructions), a k tile of a workgroup alone, and the rest of a workgroup by
// epilogue.
struct TileCost {
  int bm, bn, per_cu;
  double k[2], alone, rest[3];  // rest: STORE, GATE, GRAD
};
enum { BIG = 0, MID = 1, SMALL = 2, CONFIGS = 3 };
constexpr int64_t CUS = 256;

// bfloat16: 256 x 256 by eight waves of 128 x 64, whose LDS reads (96 bytes a
// clock at the matrix unit's full rate) stay below the CU's 128 (four waves of 128 x 128
// read 64, but nothing hides their waits: 5.39 ms against 4.68 for the whole of 16,384 x
// 2048 -> 8192); 128 x 128 by four waves of 64 x 64, which take all of them (6.09 ms); 64 x
// 64 by four waves of 32 x 32.  With all later steps: 4.52 ms, 1,090 TFLOP/s.
// float32 (three planes): 256 x 128 and 128 x 128 by waves of 64 x 64 (64
// bytes a clock), 64 x 64.  8,192 x 1024 -> 4096: 3.3 ms, 1,120 TFLOP/s of bfloat16 products.
inline const TileCost* tile_costs(bool f32) {
  static const TileCost wide[CONFIGS] = {{256, 256, 1, {1.9, 1.9}, 1.65, {5, 14, 28}},
                                         {128, 128, 2, {0.56, 0.56}, 0.85, {4, 8, 14}},
                                         {64, 64, 5, {0.20, 0.30}, 0.80, {3, 6, 8}}};
  static const TileCost three[CONFIGS] = {{256, 128, 1, {2.7, 2.7}, 2.5, {6, 17, 40}},
                                          {128, 128, 1, {1.65, 1.65}, 1.5, {5, 12, 22}},
                                          {64, 64, 3, {0.50, 0.50}, 0.74, {3, 6, 9}}};
  return f32 ? three : wide;
}

// Extents and k tiles of a product, and how it is to run.
struct Shape {
  int64_t M = 0, N = 0, ktiles = 0;
  int splits = 1;
  size_t part() const { return splits == 1 ? 0 : size_t(splits) * size_t(M) * size_t(round_up(N, 4)); }
};

// The tile (the smallest with `fine`), and the parts of each product's k, of a launch of
// `count` products: the least of an estimate that counts whole rounds of a
// workgroup a CU, the longest workgroup, and the traffic of the parts' sums.
inline int plan(Shape* s, int count, bool f32, bool fine, int epilogue, bool columns) {
  const TileCost* costs = tile_costs(f32);
  double best = 1e30;
  int config = SMALL;
  int parts[GROUP_GEMMS] = {1, 1, 1};
  for (int c = fine ? SMALL : BIG; c < CONFIGS; ++c) {
    const TileCost& t = costs[c];
    const double rest = t.rest[epilogue];
    double tiles[GROUP_GEMMS], k[GROUP_GEMMS], mn[GROUP_GEMMS];
    for (int i = 0; i < count; ++i) {
      tiles[i] = double(ceil_div(s[i].M, t.bm) * ceil_div(s[i].N, t.bn));
      k[i] = double(s[i].ktiles);
      mn[i] = double(s[i].M) * double(s[i].N);
    }
    const bool may = epilogue == STORE || c != BIG;
    for (int cap = may ? 4 : 1024; cap <= 1024; cap *= 2) {
      // of the products longer than the cap, those in the mask are split
      for (int mask = 0; mask < (may ? 1 << count : 1); ++mask) {
        double groups = 0, work = 0, longest = 0, sums = 0;
        int n[GROUP_GEMMS];
        bool fresh = true;
        for (int i = 0; i < count; ++i) {
          n[i] = 1;
          if (mask >> i & 1) {
            if (s[i].ktiles <= cap) fresh = false;  // the same as without it
            n[i] = int(std::max<int64_t>(1, ceil_div(s[i].ktiles, int64_t(cap))));
          }
          const double each = k[i] / n[i];
          groups += tiles[i] * n[i];
          work += tiles[i] * n[i] * (each * t.k[columns] + rest / t.per_cu);
          longest = std::max(longest, each * t.alone + rest);
          if (n[i] > 1) sums += mn[i] * 4.0 * (2 * n[i] + 1) / 4.0e6;  // 4 TB/s
        }
        if (!fresh) continue;
        const double rounds = groups / double(CUS);
        const double full = work / double(CUS) * std::ceil(rounds) / std::max(rounds, 1e-9);
        const double time = std::max(full, longest) +
                            (sums > 0 ? sums + (epilogue == STORE ? 4.0 : 8.0) : 0.0);
        if (time < best) {
          best = time;
          config = c;
          for (int i = 0; i < count; ++i) parts[i] = n[i];
        }
      }
    }
  }
  for (int i = 0; i < count; ++i) s[i].splits = parts[i];
  return config;
}

// The block's products in a forward pass (backward = 0) or a backward one (1: G and U
// are kept, 2: made again).  `fine`: H, dG and dU in two bfloat16 planes.
struct GatedPlan {
  Shape gate, grad;         // G and U; dH
  Shape out[GROUP_GEMMS];   // Y, or dX, [dWg; dWu], dWd
  int gate_config = SMALL, grad_config = SMALL, config = SMALL;
};
inline GatedPlan plan_gated(int64_t N, int64_t D, int64_t F, int64_t O, bool f32, bool fine,
                            int backward) {
  const int64_t kt = k_extent(f32), Fp = f_padded(F);
  GatedPlan p;
  if (backward != 1) {
    p.gate = Shape{N, 2 * F, ceil_div(D, kt)};
    p.gate_config = plan(&p.gate, 1, f32, fine, GATE, false);
  }
  if (backward == 0) {
    p.out[0] = Shape{N, O, Fp / kt};
    p.config = plan(p.out, 1, f32, fine, STORE, false);
    return p;
  }
  p.out[0] = Shape{N, D, 2 * Fp / kt};
  p.out[1] = Shape{2 * Fp, D, ceil_div(N, kt)};
  p.out[2] = Shape{O, F, ceil_div(N, kt)};
  p.config = plan(p.out, GROUP_GEMMS, f32, fine, STORE, true);
  p.grad = Shape{N, F, ceil_div(O, kt)};
  p.grad_config = plan(&p.grad, 1, f32, fine, GRAD, true);
  return p;
}

// Which forward kernels a call takes: those of few rows, the narrow one, or the tiles.
//
// Few rows: 16 rows more are another pass of the matrix unit and of the rows' own loads, and the
// tiled product overtakes (2048 -> 8192 -> 2048: bfloat16 42 us at 32 rows, 61 at 64
// against the tiles' 39; float32 132 at 64 against 210).
constexpr int64_t NARROW = 64;
inline int64_t skinny_rows(bool f32) { return f32 ? 64 : 32; }
enum Way { FEW_ROWS, NARROW_WAY, TILES };
inline Way forward_way(int64_t N, int64_t D, int64_t O, bool f32, bool save) {
  if (N <= skinny_rows(f32) && !save) return FEW_ROWS;
  return D <= NARROW && O <= NARROW ? NARROW_WAY : TILES;
}

}  // namespace net
}  // namespace fd
