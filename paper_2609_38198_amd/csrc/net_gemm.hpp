// The tiled matrix product of the gated block, C[m][n] = sum_k A(m, k) B(n, k)
// on bfloat16 matrix instructions with float32 accumulators.
//
// Operands come in two orders: "rows" (k contiguous: p[m ld + k]) and "columns"
// (m contiguous: p[k ld + m]), so that no operand is ever transposed in memory:
// column tiles are transposed by the LDS read itself.  float32 operands enter
// as three bfloat16 planes (x = x0 + x1 + x2 to 24 bits; x1 is below 2^-7 of x, x2 below
// 2^-16); the six largest of the nine plane pairs are multiplied from one tile of all
// planes.  The next two, x1 y2 and x2 y1, are at most 2^-23 of x y each.  Six
// products at the bfloat16 rate are 1.5 times the float32 unit's peak.
#pragma once

#include "net_common.hpp"
#include "net_plans.hpp"

namespace fd {
namespace net {

constexpr int MAX_SEGS = 2;      // matrices contracted one after the other
template <class T>
constexpr int planes_of = sizeof(T) == 4 ? 3 : 1;
template <class T>
constexpr int k_tile = k_extent(sizeof(T) == 4);  // k of an LDS tile
constexpr int64_t MAX_LD = int64_t(1) << 22;      // a tile's byte offsets stay below 2^31

// Sixteen bytes of zeros that lanes past the end of k read.
__device__ __align__(16) const unsigned char zero_chunk[16] = {};

struct Operand {
  const bf16* p[MAX_SEGS];  // per stretch of k
  int64_t ld;               // below MAX_LD
  int64_t plane;            // elements between planes
  int64_t rows;             // m (n) extent: rows, or columns in column order (a multiple of 8)
  int64_t k;                // k extent of a stretch (row order: a multiple of 8); beyond it reads zero
};

// 64 lanes x 16 bytes into 1 KB of LDS at `to` (wave-uniform), asynchronously:
// complete after a wait for vmcnt.  In assembly, because the compiler would
// wait for every such load before any LDS read; the write to M0 needs one
// wait state before its use.  From each lane's byte offset to a uniform base, or from each
// lane's own address.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // M0 is written and said to be
__device__ __forceinline__ void lds_load16(const char* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory", "m0");
}
__device__ __forceinline__ void lds_load16(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(to), "v"(from)
               : "memory", "m0");
}
#pragma clang diagnostic pop

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

// LDS tile of EXT rows (columns) x KT of each of PL planes, moved by THREADS
// threads.
//
// Row order: EXT rows of 2 KT bytes; 16-byte chunk c of row r is at slot
// c ^ (r & 7), or c ^ (r / 2 & 3) where a row is 64 bytes, so that eight consecutive rows'
// same chunk cover all banks.
// Column order: KT rows of 2 EXT bytes; 32-byte pair p of row k is at
// p ^ s(k), s = k & 3 (and bit 3 of k as the next bit where a row has
// eight pairs or more), so that the four rows which a transposing read of 16 lanes
// takes at once lie in different banks.
template <int EXT, int KT, int PL, int THREADS, bool COL>
struct Tile {
  static constexpr int PLANE = EXT * KT * 2;
  static constexpr int BYTES = PLANE * PL;
  static constexpr int USED = PLANE / 16 < THREADS ? PLANE / 16 : THREADS;  // threads that load
  static constexpr int LOADS = PLANE / 16 / USED;     // of a thread and plane
  static constexpr int CPR = COL ? EXT / 8 : KT / 8;  // chunks per LDS row
  static_assert(USED % WAVE == 0 && PLANE % (16 * USED) == 0 && USED % CPR == 0, "whole loads");

  uint32_t off[LOADS];  // byte offset of each load from the tile's corner
  int kofs[COL ? LOADS : 1];  // k of each load (row order: the same for all)
  int64_t corner, step, plane;  // bytes from a stretch's start to the tile, to the next k tile, plane

  static __device__ __forceinline__ int row_swizzle(int r) { return KT == 64 ? r & 7 : r >> 1 & 3; }
  static __device__ __forceinline__ int col_swizzle(int k) {
    return CPR >= 16 ? ((k & 3) | ((k >> 3) & 1) << 2) : (k & 3);
  }

  // r0: the tile's first row (column) of the operand.  Rows past the edge read
  // the last one, columns past it the tile's first: those results are dropped.
  __device__ __forceinline__ void init(const Operand& op, int64_t r0) {
    const int tid = threadIdx.x;
    if (r0 >= op.rows) r0 = 0;  // a tile of padding alone
    const int left = int(min(int64_t(EXT), op.rows - r0));
    const uint32_t ld = uint32_t(op.ld);  // below MAX_LD: offsets fit 32 bits
    plane = op.plane * 2;
    corner = COL ? r0 * 2 : r0 * op.ld * 2;
    step = COL ? KT * 2 * op.ld : KT * 2;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = (tid % USED + i * USED) / CPR, slot = tid % CPR;
      if (COL) {
        const int c = (slot ^ (col_swizzle(r) << 1)) * 8;
        kofs[i] = r;
        off[i] = (uint32_t(r) * ld + uint32_t(c < left ? c : 0)) * 2;
      } else {
        const int c = (slot ^ row_swizzle(r)) * 8;
        if (i == 0) kofs[0] = c;
        off[i] = (uint32_t(min(r, left - 1)) * ld + uint32_t(c)) * 2;
      }
    }
  }
  static_assert(COL || LOADS == 1 || (USED / CPR) % 8 == 0, "one k for a thread's row loads");

  // Issues the loads of the k tile at p (uniform), of which `left` k are there.
  __device__ __forceinline__ void load(const char* p, int left, uint32_t lds) const {
    uint32_t to = __builtin_amdgcn_readfirstlane(lds + (threadIdx.x / WAVE) * (WAVE * 16));
    if (USED < THREADS && uniform(int(threadIdx.x)) >= USED) return;  // whole waves
#pragma unroll
    for (int q = 0; q < PL; ++q) {
      if (left >= KT) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) lds_load16(p, off[i], to + i * USED * 16);
      } else {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const void* from =
              kofs[COL ? i : 0] < left ? static_cast<const void*>(p + off[i]) : zero_chunk;
          lds_load16(from, to + i * USED * 16);
        }
      }
      p += plane;
      to += PLANE;
    }
  }

  // The matrix operand of 32 rows (columns) from r0 on, k step ks, of the plane at
  // lds: lane l has row l % 32, k = 16 ks + 8 (l / 32) + 0..7.
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
    const int row = r0 + l % 32, chunk = (ks * 2 + l / 32) ^ row_swizzle(l % 32);
    return *reinterpret_cast<const bf16x8*>(lds + row * (KT * 2) + chunk * 16);
  }
};

// x as three bfloat16 values that add up to it exactly: the first cut off (a
// rounded one could leave the range), the others rounded.  An infinity becomes
// a NaN.  Six instructions a value.
__device__ __forceinline__ void split3(float x, bf16& a, bf16& b, bf16& c) {
  const uint32_t top = __builtin_bit_cast(uint32_t, x) & 0xffff0000u;
  a = __builtin_bit_cast(bf16, uint16_t(top >> 16));
  const float r = x - __builtin_bit_cast(float, top);
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

// act(g) and its derivative, of pre-activations of a block of type T.
//
// SiLU's error is the exponential's argument's: |g| 2^-24 of the value far out.
//
// GELU: with x = |g| / sqrt 2, erfc(x) = exp(-x^2) t P(t), t = 1 / (1 + p x), which keeps
// its relative accuracy in the tail, where Phi(g) is that difference from one and
// nothing else.  The exponential is also the derivative's.  P and p are least-maximum fits of the
// relative error for x up to 10.2, beyond which erfc has left float32: degree 8, 4.4e-8, for float32
// (with x^2 in two words, or its rounding would be up to 1e-5 of the value: Phi to 4e-7
// from -13 on); degree 4, 4e-5, for bfloat16, whose rounding is 2^-9.
struct Act {
  float value, slope;
};
template <int ACT, class T>
__device__ __forceinline__ Act activate(float g) {
  constexpr bool FULL = sizeof(T) == 4;
  Act a;
  if (ACT == FD_ACT_SILU) {
    const float z = __builtin_amdgcn_rcpf(1.f + __expf(-g));
    a.value = g * z;
    a.slope = z * (1.f + g * (1.f - z));
  } else {
    float e, t, q;
    if (FULL) {
      const float x = fminf(fabsf(g), 20.f);  // exp(-200) is zero, and nothing overflows
      constexpr float K = 0.7213475f, K1 = 9.629815e-09f;  // log2(e) / 2 in two words
      const float hi = x * x, lo = fmaf(x, x, -hi), u = hi * K;
      const float rest = fmaf(hi, K1, fmaf(lo, K, fmaf(hi, K, -u)));
      e = __builtin_amdgcn_exp2f(-u);
      e = fmaf(-e, rest * 0.69314718f, e);
      t = __builtin_amdgcn_rcpf(fmaf(x, 0.33587572f, 1.f));
      constexpr float P[9] = {-0.04775394f, 0.26531526f, -0.5411254f, 0.42149332f, -0.09736633f,
                              0.2351757f, 0.22727302f, 0.2690432f, 0.26794523f};
      q = P[0];
#pragma unroll
      for (int i = 1; i < 9; ++i) q = fmaf(q, t, P[i]);
    } else {
      const float x = fabsf(g) * 0.70710678f;
      e = __expf(-x * x);
      t = __builtin_amdgcn_rcpf(fmaf(x, 0.525f, 1.f));
      constexpr float P[5] = {-0.17918006f, 0.4112108f, 0.15910082f, 0.31389964f, 0.29500666f};
      q = P[0];
#pragma unroll
      for (int i = 1; i < 5; ++i) q = fmaf(q, t, P[i]);
    }
    const float c = e * t * q;
    const float z = g < 0.f ? 0.5f * c : 1.f - 0.5f * c;
    a.value = g * z;
    a.slope = z + g * e * 0.39894228f;
  }
  return a;
}

struct GemmArgs {
  Operand a, b;
  const bf16* up;       // GATE: the up weights, laid out as b's
  int64_t M, N;         // extents of C (GATE: N = F)
  int segs;             // stretches of k
  int64_t ktiles;       // k tiles of a stretch
  int splits;           // parts of the k tiles, each with its own workgroups
  int64_t tiles_m, tiles_n;
  // STORE: row r of C goes to out[r / half], row r % half, if that is below
  // `rows`; where k is split, all rows of split s go to part + s M ldp
  void* out[2];
  int64_t ldo, half, rows;
  const void *bias, *R;  // of type T, or NULL
  int64_t ldr;
  float* part;
  int64_t ldp;
  // GATE, GRAD; where k is split, the blocks' raw accumulators go to part, by
  // part and block as the kept ones lie in float32, and a kernel after it does the rest
  const void *bg, *bu;  // of the block's type, or NULL
  char* saved;          // G and U by 32 x 32 blocks, or NULL
  int64_t Fp;           // F rounded up to F_PAD: the planes' row length
  bf16 *H, *dGU;        // N x Fp, N x 2 Fp, HP planes each
  int64_t hplane, gplane;  // elements between planes
  float* colsum;        // 2 Fp column sums for each row of waves of each row tile, or NULL
};

// G and U are kept for the backward pass by 32 x 32 blocks in the accumulators'
// own order, so that both sides move whole lines without a detour.  A float32
// block keeps 4-byte values; a bfloat16 block the upper three bytes of each: all
// of float32's range whatever lies beside a value, and less than 2^-15 of it cut
// off, 1/64 of what the gradients' own rounding loses, for 3/4 of the bytes of the
// backward pass's largest operand.
template <class T>
constexpr int64_t saved_block_bytes = sizeof(T) == 4 ? 8192 : 6144;

template <class T>
__device__ __forceinline__ char* saved_at(char* saved, int64_t m, int64_t f, int64_t Fp) {
  return saved + ((m / 32) * (Fp / 32) + f / 32) * saved_block_bytes<T>;
}

// One of a block's two arrays (which = 0: G, 1: U) lies in quads of 16 bytes a
// lane, quad q of lane l at 16 (64 q + l).  float32: four values each.  bfloat16:
// the upper halves of the values 0 to 7 and 8 to 15, then the third byte of each.
template <class T>
constexpr int kept_quads = sizeof(T) == 4 ? 4 : 3;
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

template <class T>
__device__ __forceinline__ void save16(char* block, int which, int lane, const floatx16& x) {
  uintx4 v[kept_quads<T>];
  const auto bits = [&](int i) { return __builtin_bit_cast(uint32_t, float(x[i])); };
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    if constexpr (sizeof(T) == 4) {
      v[i / 4] = uintx4{bits(i), bits(i + 1), bits(i + 2), bits(i + 3)};
    } else {
      // (a byte permutation takes bytes 0 to 3 of its second word as 0 to 3, of its first as 4 to 7)
      v[i / 8][i % 8 / 2] = __builtin_amdgcn_perm(bits(i + 1), bits(i), 0x07060302);
      v[i / 8][i % 8 / 2 + 1] = __builtin_amdgcn_perm(bits(i + 3), bits(i + 2), 0x07060302);
      v[kept_quads<T> - 1][i / 4] = __builtin_amdgcn_perm(bits(i + 1), bits(i), 0x0c0c0501) |
                                    __builtin_amdgcn_perm(bits(i + 3), bits(i + 2), 0x05010c0c);
    }
  }
#pragma unroll
  for (int q = 0; q < kept_quads<T>; ++q)
    *reinterpret_cast<uintx4*>(block + ((which * kept_quads<T> + q) * WAVE + lane) * 16) = v[q];
}
// The same, back: as it lies in memory (nothing waits for it yet), then widened.
template <class T>
struct Kept {
  uintx4 v[kept_quads<T>];
};
template <class T>
__device__ __forceinline__ Kept<T> load_kept(const char* block, int which, int lane) {
  Kept<T> k;
#pragma unroll
  for (int q = 0; q < kept_quads<T>; ++q)
    k.v[q] = *reinterpret_cast<const uintx4*>(block + ((which * kept_quads<T> + q) * WAVE + lane) * 16);
  return k;
}
template <class T>
__device__ __forceinline__ floatx16 widen_kept(const Kept<T>& k) {
  floatx16 x;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    uint32_t w;
    if constexpr (sizeof(T) == 4)
      w = k.v[i / 4][i % 4];
    else  // 0, the third byte, the upper half
      w = __builtin_amdgcn_perm(k.v[i / 8][i % 8 / 2], k.v[kept_quads<T> - 1][i / 4],
                                (i % 2 == 0 ? 0x0504000cu : 0x0706000cu) | uint32_t(i % 4) << 8);
    x[i] = __builtin_bit_cast(float, w);
  }
  return x;
}

// XCD-aware order: workgroups go to the 8 XCDs in turn, so each XCD gets one
// contiguous stretch of tiles; within it, groups of 8 row tiles walk the
// columns together and share their operand tiles in that XCD's L2.
__device__ __forceinline__ void place(const GemmArgs& p, int64_t id, int64_t& tm, int64_t& tn,
                                      int& split) {
  const int64_t n = p.tiles_m * p.tiles_n * p.splits;
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

// x as PL planes: rounded; rounded and the rest (16 bits or more); or all of it.
template <int PL>
__device__ __forceinline__ void to_planes(float x, bf16 (&out)[PL]) {
  if constexpr (PL == 3) {
    split3(x, out[0], out[1], out[2]);
  } else {
    out[0] = bf16(x);
    if constexpr (PL == 2) {
      const float rest = x - float(out[0]);
      out[1] = bf16(fabsf(rest) < INFINITY ? rest : 0.f);  // an infinity stays one
    }
  }
}
template <int PL>
__device__ __forceinline__ void to_planes(const float* x, bf16x8 (&out)[PL]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    bf16 v[PL];
    to_planes<PL>(x[i], v);
#pragma unroll
    for (int q = 0; q < PL; ++q) out[q][i] = v[q];
  }
}
template <int PL>
__device__ __forceinline__ void write_planes(bf16* p, int64_t plane, const float* x) {
  bf16x8 v[PL];
  to_planes<PL>(x, v);
#pragma unroll
  for (int q = 0; q < PL; ++q) *reinterpret_cast<bf16x8*>(p + q * plane) = v[q];
}

// The plane pairs of a product that are worth their time, smallest first: all
// with one plane on a side, of 3 x 3 the six largest.
template <int PLA, int PLB>
struct Pairs {
  static constexpr bool SIX = PLA == 3;
  static_assert(SIX ? PLB == 3 : PLA * PLB <= 2, "1, 2 or 3 x 3 planes");
  static constexpr int COUNT = SIX ? 6 : PLA * PLB;
  static constexpr int six_a[6] = {1, 0, 2, 0, 1, 0}, six_b[6] = {1, 2, 0, 1, 0, 0};
  static constexpr int a(int i) { return SIX ? six_a[i] : PLA == 2 ? 1 - i : 0; }
  static constexpr int b(int i) { return SIX ? six_b[i] : PLB == 2 ? 1 - i : 0; }
};

// BM x BN tile of C by WM x WN waves of (BM / WM) x (BN / WN).  The matrix
// instruction takes the n operand first, so that a lane holds four
// consecutive n of one m: fragment value i is n = 8 (i / 4) + 4 (l / 32) + i % 4,
// m = l % 32.
//
// PLA, PLB: the operands' planes; HP: those of H, dG and dU.  id: the
// workgroup's number within the product.
template <int BM, int BN, class T, int PLA, int PLB>
constexpr size_t gemm_lds = 2 * (BM * PLA + BN * PLB) * k_tile<T> * 2;

template <int BM, int BN, int WM, int WN, bool ACOL, bool BCOL, int EPI, class T, int ACT, int PLA,
          int PLB, int HP>
__device__ __forceinline__ void gemm_body(const GemmArgs& p, int64_t id, char* smem) {
  constexpr int THREADS = WM * WN * WAVE, KT = k_tile<T>;
  using P = Pairs<PLA, PLB>;
  constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
  constexpr int BH = EPI == GATE ? BN / 2 : BN;  // extent of one b operand
  using TA = Tile<BM, KT, PLA, THREADS, ACOL>;
  using TB = Tile<BH, KT, PLB, THREADS, BCOL>;
  constexpr int BUF = TA::BYTES + TB::BYTES * (EPI == GATE ? 2 : 1);
  static_assert(2 * BUF == gemm_lds<BM, BN, T, PLA, PLB>, "the launch's size");
  static_assert(EPI != GATE || FN % 2 == 0, "gate and up fragments in pairs");

  int64_t tm, tn;
  int split;
  place(p, id, tm, tn, split);
  const int64_t m0 = uniform(tm * BM), n0 = uniform(tn * BH);
  TA ta;
  TB tb;
  ta.init(p.a, m0);
  tb.init(p.b, n0);

  // where the next k tile comes from, in scalar registers
  const int64_t total = p.ktiles * p.segs;
  const int t0 = uniform(int(total * split / p.splits));
  const int tiles = uniform(int(total * (split + 1) / p.splits)) - t0;
  int seg = uniform(int(t0 / p.ktiles));
  int kt = uniform(int(t0 - seg * p.ktiles));
  const int ktiles = int(p.ktiles);
  const char *pa = nullptr, *pb = nullptr, *pb2 = nullptr;
  int lefta = 0, leftb = 0;
  auto at = [](const bf16* x, int64_t bytes) {
    return reinterpret_cast<const char*>(uniform(reinterpret_cast<int64_t>(x) + bytes));
  };
  auto enter = [&] {  // the stretch seg at k tile kt
    const int64_t b = kt * tb.step + tb.corner;
    pa = at(p.a.p[seg], kt * ta.step + ta.corner);
    pb = at(p.b.p[seg], b);
    if (EPI == GATE) pb2 = at(p.up, b);
    lefta = uniform(int(p.a.k - int64_t(kt) * KT));
    leftb = uniform(int(p.b.k - int64_t(kt) * KT));
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
      lefta -= KT;
      leftb -= KT;
    }
  };

  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
  const int wm = wave / WN, wn = wave % WN;
  // Three planes: the five smaller pairs have sums of their own, so that the
  // large one is rounded once a k step and not six times.
  floatx16 acc[FM][FN], low[P::SIX ? FM : 1][P::SIX ? FN : 1];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        acc[i][j][e] = 0.f;
        if (P::SIX) low[i][j][e] = 0.f;
      }

  // Fragments of k step ks of the tile in a buffer.  GATE: the first half of the n
  // fragments are gate columns, the others the same up columns.
  bf16x8 fa[2][PLA][FM], fb[2][PLB][FN];
  auto read = [&](int into, int buf, int ks) {
    const char* sa = smem + buf * BUF;
    const char* sb = sa + TA::BYTES;
#pragma unroll
    for (int q = 0; q < (PLA > PLB ? PLA : PLB); ++q) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
        if (q < PLA) fa[into][q][i] = TA::fragment(sa + q * TA::PLANE, wm * TM + i * 32, ks);
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        if (q >= PLB) continue;
        constexpr int HALF = EPI == GATE ? FN / 2 : FN;
        fb[into][q][j] = TB::fragment(sb + (j / HALF) * TB::BYTES + q * TB::PLANE,
                                      wn * HALF * 32 + (j % HALF) * 32, ks);
      }
    }
  };
  auto multiply = [&](int from) {
#pragma unroll
    for (int q = 0; q < P::COUNT; ++q)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          floatx16& to =
              P::SIX && q + 1 < P::COUNT ? low[P::SIX ? i : 0][P::SIX ? j : 0] : acc[i][j];
          to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[from][P::b(q)][j], fa[from][P::a(q)][i],
                                                       to, 0, 0, 0);
        }
  };
  // The scheduler's order within a step: LDS reads evenly among the products.
  auto interleave = [] {
    constexpr int READS = PLA * FM * (ACOL ? 2 : 1) + PLB * FN * (BCOL ? 2 : 1);
    constexpr int MULS = FM * FN * P::COUNT;
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
  constexpr int STEPS = KT / 16;
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
  if (P::SIX) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] += low[P::SIX ? i : 0][P::SIX ? j : 0];
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
  const int64_t nw = n0 + wn * CN;           // the wave's first column
  const int64_t nl = nw + (lane % LPR) * 8;  // the lane's, on reading back

  if (EPI == STORE && p.splits > 1) {
    float* to = p.part + split * p.M * p.ldp;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int j = 0; j < FN; ++j) put(j, acc[i][j]);
      wave_fence();
      for (int r = lane / LPR; r < 32; r += RPP) {
        const int64_t m = m0 + wm * TM + i * 32 + r;
        if (m >= p.M || nl >= p.N) continue;
        float x[8];
        get(r, x);
        store_wide<8>(to + m * p.ldp + nl, int(min(int64_t(8), p.N - nl)), x);
      }
      wave_fence();
    }
    return;
  }

  if (EPI == STORE) {
    const int valid = int(min(int64_t(8), p.N - nl));
    float bias[8];
    if (p.bias != nullptr && nl < p.N)
      load_wide<8>(static_cast<const T*>(p.bias) + nl, valid, bias);
    else
      for (int e = 0; e < 8; ++e) bias[e] = 0.f;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int j = 0; j < FN; ++j) put(j, acc[i][j]);
      wave_fence();
      for (int r = lane / LPR; r < 32; r += RPP) {
        const int64_t m = m0 + wm * TM + i * 32 + r;
        if (m >= p.M || nl >= p.N) continue;
        const int64_t row = m < p.half ? m : m - p.half;
        T* to = static_cast<T*>(p.out[m < p.half ? 0 : 1]);
        if (row >= p.rows || to == nullptr) continue;
        float x[8], y[8];
        get(r, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += bias[e];
        if (p.R != nullptr) {
          load_wide<8>(static_cast<const T*>(p.R) + m * p.ldr + nl, valid, y);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] += y[e];
        }
        store_wide<8>(to + row * p.ldo + nl, valid, x);
      }
      wave_fence();
    }
  }

  // Rows of planes from the slab.
  auto write = [&](bf16* to, int64_t ld, int64_t plane, int64_t mb) {
    for (int r = lane / LPR; r < 32; r += RPP) {
      if (mb + r >= p.M || nl >= p.Fp) continue;
      float x[8];
      get(r, x);
      write_planes<HP>(to + (mb + r) * ld + nl, plane, x);
    }
  };

  // (not of the largest tiles, whose epilogues have no register to spare)
  if (EPI != STORE && BM < 256 && p.splits > 1) {
    constexpr int MATS = EPI == GATE ? 2 : 1, HALF = FN / MATS > 0 ? FN / MATS : 1;
    const int64_t blocks = (p.M + 31) / 32 * (p.Fp / 32);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int64_t mb = m0 + wm * TM + i * 32;
      if (mb >= p.M) break;
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int64_t fb = nw + j % HALF * 32;
        if (fb >= p.Fp) continue;
        const int64_t block = split * blocks + mb / 32 * (p.Fp / 32) + fb / 32;
        char* to = reinterpret_cast<char*>(p.part + block * (MATS * 1024));
        save16<float>(to, j / HALF, lane, acc[i][j]);
      }
    }
    return;
  }

  if (EPI == GATE) {
    constexpr int HALF = FN / 2 > 0 ? FN / 2 : 1;
#pragma unroll
    for (int j = 0; j < HALF; ++j) {
      const int64_t fb = nw + j * 32;
      float bg[16], bu[16];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t f = fb + 8 * q + 4 * half32;
        const int valid = int(max(int64_t(0), min(int64_t(4), p.N - f)));
#pragma unroll
        for (int e = 0; e < 4; ++e) bg[4 * q + e] = bu[4 * q + e] = 0.f;
        if (p.bg != nullptr) load_wide<4>(static_cast<const T*>(p.bg) + f, valid, bg + 4 * q);
        if (p.bu != nullptr) load_wide<4>(static_cast<const T*>(p.bu) + f, valid, bu + 4 * q);
      }
#pragma unroll
      for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          acc[i][j][e] += bg[e];
          acc[i][(j + HALF) % FN][e] += bu[e];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int64_t mb = m0 + wm * TM + i * 32;
      if (mb >= p.M) break;
#pragma unroll
      for (int j = 0; j < HALF; ++j) {
        const int64_t fb = nw + j * 32;
        const floatx16& g = acc[i][j];
        const floatx16& u = acc[i][(j + HALF) % FN];
        if (p.saved != nullptr && fb < p.Fp) {
          char* block = saved_at<T>(p.saved, mb, fb, p.Fp);
          save16<T>(block, 0, lane, g);
          save16<T>(block, 1, lane, u);
        }
        if (p.H == nullptr) continue;
        floatx16 h;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const bool there = fb + 8 * (e / 4) + 4 * half32 + e % 4 < p.N;
          h[e] = there ? activate<ACT, T>(g[e]).value * u[e] : 0.f;
        }
        put(j, h);
      }
      if (p.H == nullptr) continue;
      wave_fence();
      write(p.H, p.Fp, p.hplane, mb);
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
      floatx16 v[3][FN];  // dG, dU, H
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int64_t fb = nw + j * 32;
        if (fb < p.Fp) {
          const char* block = saved_at<T>(p.saved, mb, fb, p.Fp);
          const floatx16 g = widen_kept(load_kept<T>(block, 0, lane));
          const floatx16 u = widen_kept(load_kept<T>(block, 1, lane));
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const bool there = live && fb + 8 * (e / 4) + 4 * half32 + e % 4 < p.N;
            const Act a = activate<ACT, T>(g[e]);
            const float dh = acc[i][j][e];
            v[0][j][e] = there ? dh * u[e] * a.slope : 0.f;
            v[1][j][e] = there ? dh * a.value : 0.f;
            v[2][j][e] = there ? a.value * u[e] : 0.f;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[0][j][e] = v[1][j][e] = v[2][j][e] = 0.f;
        }
      }
#pragma unroll
      for (int what = 0; what < 3; ++what) {
#pragma unroll
        for (int j = 0; j < FN; ++j) put(j, v[what][j]);
        wave_fence();
        if (what < 2 && p.colsum != nullptr && lane < CN)
          for (int r = 0; r < 32; ++r)
#pragma unroll
            for (int c = 0; c < SC; ++c)
              sums[what][c] += *reinterpret_cast<const float*>(slab + r * PITCH + (lane + c * WAVE) * 4);
        if (what == 2) write(p.H, p.Fp, p.hplane, mb);
        else write(p.dGU + what * p.Fp, 2 * p.Fp, p.gplane, mb);
        wave_fence();
      }
    }
    if (p.colsum != nullptr && lane < CN) {
#pragma unroll
      for (int c = 0; c < SC; ++c) {
        const int64_t f = nw + lane + c * WAVE;
        if (f >= p.Fp) continue;
        float* s = p.colsum + (tm * WM + wm) * 2 * p.Fp + f;
        s[0] = sums[0][c];
        s[p.Fp] = sums[1][c];
      }
    }
  }
}

template <int BM, int BN, int WM, int WN, bool ACOL, bool BCOL, int EPI, class T, int ACT, int PLA,
          int PLB, int HP>
__global__ __launch_bounds__(WM * WN * WAVE) void gemm_kernel(GemmArgs p) {
  extern __shared__ __align__(1024) char smem[];
  gemm_body<BM, BN, WM, WN, ACOL, BCOL, EPI, T, ACT, PLA, PLB, HP>(p, blockIdx.x, smem);
}

// The backward pass's last products, which do not depend on each other, in one
// launch: the workgroups of one fill what another leaves idle.
struct GemmGroup {
  GemmArgs g[GROUP_GEMMS];
  bool acol[GROUP_GEMMS];          // a in column order (b always is)
  bool inner[GROUP_GEMMS];         // b, and not a, has HP planes
  int64_t first[GROUP_GEMMS + 1];  // a product's first workgroup
  int count;
};

template <int BM, int BN, int WM, int WN, class T, int HP>
__global__ __launch_bounds__(WM * WN * WAVE) void gemm_group_kernel(GemmGroup s) {
  extern __shared__ __align__(1024) char smem[];
  int i = 0;
  while (i + 1 < s.count && s.first[i + 1] <= int64_t(blockIdx.x)) ++i;
  const int64_t id = int64_t(blockIdx.x) - s.first[i];
  constexpr int PL = planes_of<T>;
  if (!s.acol[i])
    gemm_body<BM, BN, WM, WN, false, true, STORE, T, 0, HP, PL, HP>(s.g[i], id, smem);
  else if (HP == PL || !s.inner[i])
    gemm_body<BM, BN, WM, WN, true, true, STORE, T, 0, HP, PL, HP>(s.g[i], id, smem);
  else if constexpr (HP != PL)
    gemm_body<BM, BN, WM, WN, true, true, STORE, T, 0, PL, HP, HP>(s.g[i], id, smem);
}

// The rest of a GATE or GRAD product whose k is split: a wave to a 32 x 32 block
// adds the parts in their order and goes on as the product's own epilogue does.
template <int EPI, class T, int ACT, int HP>
__global__ __launch_bounds__(256) void finish_kernel(GemmArgs p) {
  constexpr int MATS = EPI == GATE ? 2 : 1;
  const int lane = threadIdx.x % WAVE, half32 = lane / 32;
  const int64_t across = p.Fp / 32, blocks = (p.M + 31) / 32 * across;
  const int64_t at = int64_t(blockIdx.x) * (256 / WAVE) + threadIdx.x / WAVE;
  if (at >= blocks) return;
  const int64_t mb = at / across * 32, fb = at % across * 32, m = mb + lane % 32;
  floatx16 x[2];
#pragma unroll
  for (int w = 0; w < MATS; ++w) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[w][e] = 0.f;
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s)
      x[w] += widen_kept(load_kept<float>(
          reinterpret_cast<const char*>(p.part + (s * blocks + at) * (MATS * 1024)), w, lane));
  }
  floatx16 out[3];
  if (EPI == GATE) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t f = fb + 8 * q + 4 * half32;
      const int valid = int(max(int64_t(0), min(int64_t(4), p.N - f)));
      float bg[4] = {0.f, 0.f, 0.f, 0.f}, bu[4] = {0.f, 0.f, 0.f, 0.f};
      if (p.bg != nullptr) load_wide<4>(static_cast<const T*>(p.bg) + f, valid, bg);
      if (p.bu != nullptr) load_wide<4>(static_cast<const T*>(p.bu) + f, valid, bu);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * q + e;
        x[0][i] += bg[e];
        x[1][i] += bu[e];
        out[2][i] = e < valid ? activate<ACT, T>(x[0][i]).value * x[1][i] : 0.f;
      }
    }
    if (p.saved != nullptr) {
      char* block = saved_at<T>(p.saved, mb, fb, p.Fp);
      save16<T>(block, 0, lane, x[0]);
      save16<T>(block, 1, lane, x[1]);
    }
  } else {
    const char* block = saved_at<T>(p.saved, mb, fb, p.Fp);
    const floatx16 g = widen_kept(load_kept<T>(block, 0, lane));
    const floatx16 u = widen_kept(load_kept<T>(block, 1, lane));
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t f = fb + 8 * (e / 4) + 4 * half32 + e % 4;
      const bool there = m < p.M && f < p.N;
      const Act a = activate<ACT, T>(g[e]);
      const float dh = x[0][e];
      out[0][e] = there ? dh * u[e] * a.slope : 0.f;
      out[1][e] = there ? dh * a.value : 0.f;
      out[2][e] = there ? a.value * u[e] : 0.f;
      if (p.colsum != nullptr) {  // a row of sums for each 32 rows
        const float sg = lane_sum<32>(out[0][e]), su = lane_sum<32>(out[1][e]);
        if (lane % 32 == 0) {
          p.colsum[mb / 32 * 2 * p.Fp + f] = sg;
          p.colsum[mb / 32 * 2 * p.Fp + p.Fp + f] = su;
        }
      }
    }
  }
  if (m >= p.M) return;
#pragma unroll
  for (int w = EPI == GATE ? 2 : 0; w < 3; ++w) {
    if (w == 2 && p.H == nullptr) continue;
    bf16* to = w == 2 ? p.H + m * p.Fp : p.dGU + m * 2 * p.Fp + w * p.Fp;
    const int64_t plane = w == 2 ? p.hplane : p.gplane;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      bf16x4 v[HP];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bf16 y[HP];
        to_planes<HP>(out[w][4 * q + e], y);
#pragma unroll
        for (int k = 0; k < HP; ++k) v[k][e] = y[k];
      }
#pragma unroll
      for (int k = 0; k < HP; ++k)
        *reinterpret_cast<bf16x4*>(to + k * plane + fb + 8 * q + 4 * half32) = v[k];
    }
  }
}

}  // namespace net
}  // namespace fd
