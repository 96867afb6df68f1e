// The tiled matrix product of the gated block, C[m][n] = sum_k A(m, k) B(n, k)
// on bfloat16 matrix instructions with float32 accumulators.
//
// Operands come in two orders: "rows" (k contiguous: p[m ld + k]) and "columns"
// (m contiguous: p[k ld + m]), so that no operand is ever transposed in memory:
// column tiles are transposed by the LDS read itself.  float32 operands enter
// as three bfloat16 planes (x = x0 + x1 + x2 to 24 bits) and the contraction
// runs over the six plane pairs whose product is above 2^-24 of x y, as if
// they were further stretches of k.
#pragma once

#include "net_common.hpp"

namespace fd {
namespace net {

constexpr int BK = 64;           // k of a tile: 128 bytes of a row, one cache line
constexpr int MAX_SEGS = 12;     // stretches of k: two matrices x six plane pairs
constexpr int PLANES = 3;
constexpr int PAIRS = 6;
constexpr int64_t MAX_LD = int64_t(1) << 22;  // a tile's byte offsets stay below 2^31

// Sixteen bytes of zeros that lanes past the end of k read.
__device__ __align__(16) const unsigned char zero_chunk[16] = {};

// One operand: up to two matrices (gate and up weights in the forward product).
struct Operand {
  const bf16* p[MAX_SEGS];  // per stretch of k
  int64_t ld;               // below MAX_LD
  int64_t rows;             // m (n) extent: rows, or columns in column order (a multiple of 8)
  int64_t k;                // k extent of a stretch (row order: a multiple of 8); beyond it reads zero
};

// 64 lanes x 16 bytes into 1 KB of LDS at `to` (wave-uniform), asynchronously:
// complete after a wait for vmcnt.  In assembly, because the compiler would
// wait for every such load before any LDS read; the write to M0 needs one
// wait state before its use.  From each lane's byte offset to a uniform base, or from each
// lane's own address.
__device__ __forceinline__ void lds_load16(const char* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}
__device__ __forceinline__ void lds_load16(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(to), "v"(from)
               : "memory");
}

// A value that is the same in every lane, in a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return int64_t(uint64_t(uint32_t(uniform(int(x >> 32)))) << 32 | uint32_t(uniform(int(x))));
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)p));
}

typedef short shortx4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bf16x4 lds_read_transposed(const char* p) {
  typedef __attribute__((address_space(3))) shortx4* Ptr;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)p));
}

// LDS tile of EXT rows (columns) x BK, moved by THREADS threads.
//
// Row order: EXT rows of 128 bytes; 16-byte chunk c of row r is at slot
// c ^ (r & 7), so that eight consecutive rows' same chunk cover all banks.
// Column order: BK rows of 2 EXT bytes; 32-byte pair p of row k is at
// p ^ s(k), s = k & 3 (and bit 3 of k as the next bit where a row has
// eight pairs or more), so that the four rows which a transposing read of 16 lanes
// takes at once lie in different banks.
template <int EXT, int THREADS, bool COL>
struct Tile {
  static constexpr int BYTES = EXT * BK * 2;
  static constexpr int LOADS = BYTES / 16 / THREADS;  // of a thread
  static constexpr int CPR = COL ? EXT / 8 : 8;       // chunks per LDS row
  static_assert(BYTES % (16 * THREADS) == 0, "whole loads");
  static_assert((THREADS / CPR) % 8 == 0, "whole rows");

  uint32_t off[LOADS];  // byte offset of each load from the tile's corner
  int kofs;             // row order: k of this thread's chunk; column order: of its first load
  int64_t corner, step; // bytes from a stretch's start to the tile, and to the next k tile

  static __device__ __forceinline__ int swizzle(int k) {
    return CPR >= 16 ? ((k & 3) | ((k >> 3) & 1) << 2) : (k & 3);
  }

  // r0: the tile's first row (column) of the operand.  Rows past the edge read
  // the last one, columns past it the tile's first: those results are dropped.
  __device__ __forceinline__ void init(const Operand& op, int64_t r0) {
    const int tid = threadIdx.x;
    const int left = int(min(int64_t(EXT), op.rows - r0));
    const uint32_t ld = uint32_t(op.ld);  // below MAX_LD: offsets fit 32 bits
    if (COL) {
      kofs = tid / CPR;
      corner = r0 * 2;
      step = BK * 2 * op.ld;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int k = kofs + i * (THREADS / CPR);
        const int c = ((tid % CPR) ^ (swizzle(k) << 1)) * 8;
        off[i] = (uint32_t(k) * ld + uint32_t(c < left ? c : 0)) * 2;
      }
    } else {
      const int r = tid / 8;
      kofs = ((tid % 8) ^ (r & 7)) * 8;
      corner = r0 * op.ld * 2;
      step = BK * 2;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = min(r + i * (THREADS / 8), left - 1);
        off[i] = (uint32_t(row) * ld + uint32_t(kofs)) * 2;
      }
    }
  }

  // Issues the loads of the k tile at p (uniform), of which `left` k are there.
  __device__ __forceinline__ void load(const char* p, int left, uint32_t lds) const {
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (threadIdx.x / WAVE) * (WAVE * 16));
    if (left >= BK) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) lds_load16(p, off[i], to + i * THREADS * 16);
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int at = COL ? kofs + i * (THREADS / CPR) : kofs;
        const void* from = at < left ? static_cast<const void*>(p + off[i]) : zero_chunk;
        lds_load16(from, to + i * THREADS * 16);
      }
    }
  }

  // The matrix operand of 32 rows (columns) from r0 on, k step ks: lane l has row
  // l % 32, k = 16 ks + 8 (l / 32) + 0..7.
  static __device__ __forceinline__ bf16x8 fragment(const char* lds, int r0, int ks) {
    const int l = threadIdx.x % WAVE;
    if (COL) {
      const int group = l / 16, j = l % 16;
      const int s = CPR >= 16 ? ((j / 4) | (group >> 1) << 2) : (j / 4);
      const int pair = (r0 / 16 + (group & 1)) ^ s;
      const char* p = lds + (ks * 16 + (group >> 1) * 8 + j / 4) * (EXT * 2) + pair * 32 + (j % 4) * 8;
      const bf16x4 lo = lds_read_transposed(p), hi = lds_read_transposed(p + 4 * EXT * 2);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    const int row = r0 + l % 32, chunk = (ks * 2 + l / 32) ^ (l & 7);
    return *reinterpret_cast<const bf16x8*>(lds + row * (BK * 2) + chunk * 16);
  }
};

// x as three bfloat16 values that add up to it; a value that is not finite is
// the first one's alone.
__device__ __forceinline__ void split3(float x, bf16& a, bf16& b, bf16& c) {
  a = bf16(x);
  if (!(fabsf(float(a)) < INFINITY))  // rounded up past the largest, or not finite
    a = __builtin_bit_cast(bf16, uint16_t(__builtin_bit_cast(uint32_t, x) >> 16 |
                                          (x != x ? 0x40u : 0u)));
  const float fa = float(a);
  const float r = fabsf(fa) < INFINITY ? x - fa : 0.f;
  b = bf16(r);
  c = bf16(r - float(b));
}

// Hides a value's round trip through LDS from reordering: what one lane of the
// wave wrote, another reads (LDS serves a wave in order).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// act(g) and its derivative.
struct Act {
  float value, slope;
};
template <int ACT>
__device__ __forceinline__ Act activate(float g) {
  Act a;
  if (ACT == FD_ACT_SILU) {
    const float z = __builtin_amdgcn_rcpf(1.f + __expf(-g));
    a.value = g * z;
    a.slope = z * (1.f + g * (1.f - z));
  } else {
    // erfc by Hastings' rational fit (Abramowitz and Stegun 7.1.26, absolute
    // error 1.5e-7), whose exponential is also the derivative's
    const float x = fabsf(g) * 0.70710678f;
    const float e = __expf(-x * x);
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * x);
    const float c = e * t *
                    (0.254829592f +
                     t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    const float z = g < 0.f ? 0.5f * c : 1.f - 0.5f * c;
    a.value = g * z;
    a.slope = z + g * e * 0.39894228f;
  }
  return a;
}

// What a product does with its accumulators.
enum Epilogue {
  STORE = 0,  // C (+ bias + R) in T, or a split's float32 partial sums
  GATE = 1,   // B is [Wg; Wu]: H = act(G) U as planes, G and U kept where wanted
  GRAD = 2    // C is dH: dG, dU, H as planes from the kept G and U, column sums
};

struct GemmArgs {
  Operand a, b, b2;     // b2: GATE, the up weights
  int64_t M, N;         // extents of C (GATE: N = F)
  int segs;             // stretches of k
  int64_t ktiles;       // k tiles of a stretch
  int splits;           // parts of the k tiles, each with its own workgroups
  int64_t tiles_m, tiles_n;
  // STORE: row r of C goes to out[r / half], row r % half, if that is below `rows`
  void* out[2];
  int64_t ldo, half, rows;
  const void *bias, *R;  // of type T, or NULL
  int64_t ldr;
  // GATE, GRAD
  const void *bg, *bu;  // of the block's type, or NULL
  float* saved;         // G and U in fragment order, or NULL
  int64_t Fp;           // F rounded up to BK: the planes' row length
  bf16 *H, *dGU;        // N x Fp, N x 2 Fp
  int64_t hplane, gplane;  // elements between planes
  float* colsum;        // 2 Fp column sums for each row of waves of each row tile, or NULL
  int act;
};

// Where a 32 x 32 block of G starts in the kept buffer (U follows 1,024 floats
// later): lane l's values 4 i .. 4 i + 3 are at (64 i + l) 4, 16 bytes a lane.
__device__ __forceinline__ int64_t saved_block(int64_t m, int64_t f, int64_t Fp) {
  return ((m / 32) * (Fp / 32) + f / 32) * 2048;
}

// XCD-aware order: workgroups go to the 8 XCDs in turn, so each XCD gets one
// contiguous stretch of tiles; within it, groups of 8 row tiles walk the
// columns together and share their operand tiles in that XCD's L2.
__device__ __forceinline__ void place(const GemmArgs& p, int64_t& tm, int64_t& tn, int& split) {
  const int64_t n = gridDim.x, id = blockIdx.x;
  const int64_t q = n / 8, r = n % 8, x = id % 8;
  int64_t at = (x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q) + id / 8;
  const int64_t per = p.tiles_m * p.tiles_n;
  split = int(at / per);
  at -= split * per;
  constexpr int64_t GM = 8;
  const int64_t band = at / (GM * p.tiles_n), first = band * GM;
  const int64_t high = min(GM, p.tiles_m - first);
  at -= band * GM * p.tiles_n;
  tm = first + at % high;
  tn = at / high;
}

template <class T>
__device__ __forceinline__ void write_planes(bf16* p, int64_t plane, const float* x) {
  bf16x8 a, b, c;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (sizeof(T) == 4) {
      bf16 u, v, w;
      split3(x[i], u, v, w);
      a[i] = u;
      b[i] = v;
      c[i] = w;
    } else {
      a[i] = bf16(x[i]);
    }
  }
  *reinterpret_cast<bf16x8*>(p) = a;
  if (sizeof(T) == 4) {
    *reinterpret_cast<bf16x8*>(p + plane) = b;
    *reinterpret_cast<bf16x8*>(p + 2 * plane) = c;
  }
}

// BM x BN tile of C by WM x WN waves of (BM / WM) x (BN / WN).  The matrix
// instruction takes the n operand first, so that a lane holds four
// consecutive n of one m: fragment value i is n = 8 (i / 4) + 4 (l / 32) + i % 4,
// m = l % 32.
template <int BM, int BN, int WM, int WN, bool ACOL, bool BCOL, int EPI, class T, int ACT>
__global__ __launch_bounds__(WM * WN * WAVE) void gemm_kernel(GemmArgs p) {
  constexpr int THREADS = WM * WN * WAVE;
  constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
  constexpr int BH = EPI == GATE ? BN / 2 : BN;  // extent of one b operand
  using TA = Tile<BM, THREADS, ACOL>;
  using TB = Tile<BH, THREADS, BCOL>;
  constexpr int BUF = TA::BYTES + BN * BK * 2;
  static_assert(EPI != GATE || FN % 2 == 0, "gate and up fragments in pairs");
  extern __shared__ __align__(1024) char smem[];

  int64_t tm, tn;
  int split;
  place(p, tm, tn, split);
  const int64_t m0 = uniform(tm * BM), n0 = uniform(tn * BH);
  TA ta;
  TB tb;
  ta.init(p.a, m0);
  tb.init(p.b, n0);  // GATE: the up weights have the same shape

  // where the next k tile comes from, in scalar registers
  const int64_t total = p.ktiles * p.segs;
  const int t0 = uniform(int(total * split / p.splits));
  const int tiles = uniform(int(total * (split + 1) / p.splits)) - t0;
  int seg = uniform(int(t0 / p.ktiles));
  int kt = uniform(int(t0 - seg * p.ktiles));
  const int ktiles = int(p.ktiles);
  const char *pa = nullptr, *pb = nullptr, *pb2 = nullptr;
  int lefta = 0, leftb = 0;
  auto enter = [&] {  // the stretch seg at k tile kt
    const int64_t a = kt * ta.step + ta.corner, b = kt * tb.step + tb.corner;
    pa = reinterpret_cast<const char*>(uniform(reinterpret_cast<int64_t>(p.a.p[seg]) + a));
    pb = reinterpret_cast<const char*>(uniform(reinterpret_cast<int64_t>(p.b.p[seg]) + b));
    if (EPI == GATE)
      pb2 = reinterpret_cast<const char*>(uniform(reinterpret_cast<int64_t>(p.b2.p[seg]) + b));
    lefta = uniform(int(p.a.k - int64_t(kt) * BK));
    leftb = uniform(int(p.b.k - int64_t(kt) * BK));
  };
  const uint32_t base = lds_address(smem);
  auto issue = [&](uint32_t lds) {
    ta.load(pa, lefta, lds);
    tb.load(pb, leftb, lds + TA::BYTES);
    if (EPI == GATE) tb.load(pb2, leftb, lds + TA::BYTES + TB::BYTES);
    if (++kt == ktiles) {
      kt = 0;
      if (++seg < p.segs) enter();
    } else {
      pa += ta.step;
      pb += tb.step;
      if (EPI == GATE) pb2 += tb.step;
      lefta -= BK;
      leftb -= BK;
    }
  };

  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
  const int wm = wave / WN, wn = wave % WN;
  // first LDS row of n fragment f
  auto brow = [&](int f) {
    if (EPI == GATE)
      return (f < FN / 2 ? 0 : BN / 2) + wn * (TN / 2) + (f % (FN / 2 > 0 ? FN / 2 : 1)) * 32;
    return wn * TN + f * 32;
  };
  floatx16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // Fragments of k step ks of the tile in a buffer.
  bf16x8 fa[2][FM], fb[2][FN];
  auto read = [&](int into, int buf, int ks) {
    const char* sa = smem + buf * BUF;
    const char* sb = sa + TA::BYTES;
#pragma unroll
    for (int i = 0; i < FM; ++i) fa[into][i] = TA::fragment(sa, wm * TM + i * 32, ks);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      if (EPI == GATE && j >= FN / 2)
        fb[into][j] = TB::fragment(sb + TB::BYTES, brow(j) - BN / 2, ks);
      else
        fb[into][j] = TB::fragment(sb, brow(j), ks);
    }
  };
  auto multiply = [&](int from) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[from][j], fa[from][i], acc[i][j], 0, 0, 0);
  };

  // The scheduler's order within a step: LDS reads evenly among the products.
  auto interleave = [] {
    constexpr int READS = FM * (ACOL ? 2 : 1) + FN * (BCOL ? 2 : 1), MULS = FM * FN;
#pragma unroll
    for (int i = 0; i < MULS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, (READS + MULS - 1) / MULS, 0);
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    }
  };

  // Two LDS buffers and two sets of fragments.  The fragments of a k step are
  // read while the matrix unit works on the step before; at a tile's last step
  // every wave has its last fragments of the tile, so one barrier both shows the
  // next tile (loaded during this one) and frees this buffer for the tile after.
  constexpr int STEPS = BK / 16;
  static_assert(STEPS % 2 == 0, "the fragment sets alternate");
  if (tiles > 0) {
    enter();
    issue(base);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (tiles > 1) issue(base + BUF);
    read(0, 0, 0);
  }
  for (int t = 0; t < tiles; ++t) {
    const int cur = t & 1;
#pragma unroll
    for (int ks = 0; ks < STEPS; ++ks) {
      if (ks + 1 < STEPS) {
        read((ks + 1) & 1, cur, ks + 1);
      } else if (t + 1 < tiles) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(0, cur ^ 1, 0);
        if (t + 2 < tiles) issue(base + cur * BUF);
      }
      multiply(ks & 1);
      interleave();
    }
  }
  __syncthreads();  // the buffers become the waves' staging slabs

  // A slab holds 32 rows of CN columns in float32, rows 16 bytes apart from
  // a multiple of all banks; lanes then read back eight columns of a row each, so that
  // global rows are written in whole lines.
  constexpr int CN = EPI == GATE ? TN / 2 : TN;
  constexpr int PITCH = CN * 4 + 16;
  constexpr int LPR = CN / 8, RPP = WAVE / LPR;  // lanes of a row, rows of a pass
  char* slab = smem + wave * (32 * PITCH);
  const int half32 = lane / 32;
  auto put = [&](int j, const floatx16& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      floatx4 q = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
      *reinterpret_cast<floatx4*>(slab + (lane % 32) * PITCH + (j * 32 + 8 * i + 4 * half32) * 4) = q;
    }
  };
  auto get = [&](int row, float* x) {
    const char* s = slab + row * PITCH + (lane % LPR) * 32;
    const floatx4 a = *reinterpret_cast<const floatx4*>(s);
    const floatx4 b = *reinterpret_cast<const floatx4*>(s + 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  };
  const int64_t nw = n0 + wn * CN;          // the wave's first column
  const int64_t nl = nw + (lane % LPR) * 8;  // the lane's, on reading back

  if (EPI == STORE) {
    float bias[8];
    if (p.bias != nullptr && nl < p.N)
      load_wide<8>(static_cast<const T*>(p.bias) + nl, int(min(int64_t(8), p.N - nl)), bias);
    else
      for (int e = 0; e < 8; ++e) bias[e] = 0.f;
    T* o0 = static_cast<T*>(p.out[0]);
    T* o1 = static_cast<T*>(p.out[1]);
    if (p.splits > 1) o0 += split * p.M * p.ldo;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int j = 0; j < FN; ++j) put(j, acc[i][j]);
      wave_fence();
      for (int r = lane / LPR; r < 32; r += RPP) {
        const int64_t m = m0 + wm * TM + i * 32 + r;
        if (m >= p.M || nl >= p.N) continue;
        const int64_t row = m < p.half ? m : m - p.half;
        if (row >= p.rows) continue;
        const int valid = int(min(int64_t(8), p.N - nl));
        float x[8], y[8];
        get(r, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += bias[e];
        if (p.R != nullptr) {
          load_wide<8>(static_cast<const T*>(p.R) + m * p.ldr + nl, valid, y);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] += y[e];
        }
        store_wide<8>((m < p.half ? o0 : o1) + row * p.ldo + nl, valid, x);
      }
      wave_fence();
    }
  }

  if (EPI == GATE) {
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int64_t mb = m0 + wm * TM + i * 32;
#pragma unroll
      for (int j = 0; j < FN / 2; ++j) {
        const int64_t fb = nw + j * 32;
        floatx16 h;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t f = fb + 8 * q + 4 * half32;
          const int valid = int(max(int64_t(0), min(int64_t(4), p.N - f)));
          float bg[4] = {0.f, 0.f, 0.f, 0.f}, bu[4] = {0.f, 0.f, 0.f, 0.f};
          if (p.bg != nullptr) load_wide<4>(static_cast<const T*>(p.bg) + f, valid, bg);
          if (p.bu != nullptr) load_wide<4>(static_cast<const T*>(p.bu) + f, valid, bu);
          floatx4 g, u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            g[e] = acc[i][j][4 * q + e] + bg[e];
            u[e] = acc[i][j + FN / 2][4 * q + e] + bu[e];
            h[4 * q + e] = e < valid ? activate<ACT>(g[e]).value * u[e] : 0.f;
          }
          if (p.saved != nullptr && mb < p.M && fb < p.Fp) {
            float* s = p.saved + saved_block(mb, fb, p.Fp) + (q * WAVE + lane) * 4;
            *reinterpret_cast<floatx4*>(s) = g;
            *reinterpret_cast<floatx4*>(s + 1024) = u;
          }
        }
        put(j, h);
      }
      if (p.H == nullptr) continue;
      wave_fence();
      for (int r = lane / LPR; r < 32; r += RPP) {
        if (mb + r >= p.M || nl >= p.Fp) continue;
        float x[8];
        get(r, x);
        write_planes<T>(p.H + (mb + r) * p.Fp + nl, p.hplane, x);
      }
      wave_fence();
    }
  }

  if (EPI == GRAD) {
    constexpr int SC = (CN + WAVE - 1) / WAVE;  // columns that a lane sums
    float sums[2][SC] = {};
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int64_t mb = m0 + wm * TM + i * 32;
      if (mb >= p.M) break;
      const bool live = mb + lane % 32 < p.M;
#pragma unroll
      for (int what = 0; what < 3; ++what) {  // dG, dU, H
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const int64_t fb = nw + j * 32;
          floatx16 v;
          if (fb < p.Fp) {
            const float* s = p.saved + saved_block(mb, fb, p.Fp) + lane * 4;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const floatx4 g = *reinterpret_cast<const floatx4*>(s + q * WAVE * 4);
              const floatx4 u = *reinterpret_cast<const floatx4*>(s + 1024 + q * WAVE * 4);
              const int64_t f = fb + 8 * q + 4 * half32;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const Act a = activate<ACT>(g[e]);
                const float dh = acc[i][j][4 * q + e];
                const float x = what == 0 ? dh * u[e] * a.slope : what == 1 ? dh * a.value : a.value * u[e];
                v[4 * q + e] = live && f + e < p.N ? x : 0.f;
              }
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = 0.f;
          }
          put(j, v);
        }
        wave_fence();
        if (what < 2 && p.colsum != nullptr && lane < CN)
          for (int r = 0; r < 32; ++r)
#pragma unroll
            for (int c = 0; c < SC; ++c)
              sums[what][c] += *reinterpret_cast<const float*>(slab + r * PITCH + (lane + c * WAVE) * 4);
        bf16* to = what == 2 ? p.H : p.dGU + (what == 1 ? p.Fp : 0);
        const int64_t ld = what == 2 ? p.Fp : 2 * p.Fp, plane = what == 2 ? p.hplane : p.gplane;
        for (int r = lane / LPR; r < 32; r += RPP) {
          if (mb + r >= p.M || nl >= p.Fp) continue;
          float x[8];
          get(r, x);
          write_planes<T>(to + (mb + r) * ld + nl, plane, x);
        }
        wave_fence();
      }
    }
#pragma unroll
    for (int c = 0; c < SC; ++c) {
      const int64_t f = nw + lane + c * WAVE;
      if (p.colsum != nullptr && lane < CN && f < p.Fp) {
        float* s = p.colsum + (tm * WM + wm) * 2 * p.Fp + f;
        s[0] = sums[0][c];
        s[p.Fp] = sums[1][c];
      }
    }
  }
}

}  // namespace net
}  // namespace fd
