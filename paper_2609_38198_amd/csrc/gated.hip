// The gated feed-forward block, forward and backward.
#include <algorithm>

#include "fd_guard.hpp"
#include "fd_solver.hpp"
#include "net_gemm.hpp"

namespace fd {
namespace net {
namespace {

constexpr int GROUP = 256;

// ---------------------------------------------------------------- packing
// A matrix as bfloat16 planes with rows of a multiple of eight elements, zeros
// past the end: what the product's 16-byte loads need of operands that are
// float32, odd in width or not 16-byte aligned.
struct PackJob {
  const void* src;
  int64_t ld, rows, cols, ldp;  // ldp: columns rounded up to 8
  bf16* dst;
  int64_t plane;
  int64_t first;                // the job's first workgroup
};
constexpr int PACK_JOBS = 5;
struct PackJobs {
  PackJob j[PACK_JOBS];
  int count = 0;
  int64_t groups = 0;
};

template <class T>
__global__ __launch_bounds__(GROUP) void pack_kernel(PackJobs jobs) {
  int i = 0;
  while (i + 1 < jobs.count && jobs.j[i + 1].first <= int64_t(blockIdx.x)) ++i;
  const PackJob& job = jobs.j[i];
  const int64_t at = (int64_t(blockIdx.x) - job.first) * GROUP + threadIdx.x;
  const int64_t per = job.ldp / 8, row = at / per, col = (at - row * per) * 8;
  if (row >= job.rows) return;
  float x[8];
  load_wide<8>(static_cast<const T*>(job.src) + row * job.ld + col,
               int(min(int64_t(8), job.cols - col)), x);
  write_planes<T>(job.dst + row * job.ldp + col, job.plane, x);
}

// ---------------------------------------------------------------- sums
// Partial column sums of a matrix: workgroup (x, y) adds rows y, y + gridDim.y,
// ... of columns x; in the order of the rows, so the total's order is fixed.
template <class T>
__global__ __launch_bounds__(GROUP) void column_sum_kernel(const T* A, int64_t lda, int64_t rows,
                                                           int64_t cols, float* part) {
  __shared__ float sums[4][WAVE];
  const int c = threadIdx.x % WAVE, r = threadIdx.x / WAVE;
  const int64_t col = int64_t(blockIdx.x) * WAVE + c;
  float s = 0.f;
  if (col < cols)
    for (int64_t i = int64_t(blockIdx.y) * 4 + r; i < rows; i += int64_t(gridDim.y) * 4)
      s += widen(A[i * lda + col]);
  sums[r][c] = s;
  __syncthreads();
  if (r == 0 && col < cols) {
    for (int i = 1; i < 4; ++i) s += sums[i][c];
    part[int64_t(blockIdx.y) * cols + col] = s;
  }
}

// Sums over `rows` rows of float32 partial sums, ld apart; column c of the
// first `valid` of every `width` goes to out[c / width].
template <class T>
__global__ __launch_bounds__(GROUP) void reduce_columns_kernel(const float* part, int64_t rows,
                                                               int64_t ld, int64_t width,
                                                               int64_t valid, T* out0, T* out1) {
  __shared__ float sums[16][17];
  const int c = threadIdx.x % 16, r = threadIdx.x / 16;
  const int64_t col = int64_t(blockIdx.x) * 16 + c;
  float s = 0.f;
  if (col < ld)
    for (int64_t i = r; i < rows; i += 16) s += part[i * ld + col];
  sums[r][c] = s;
  __syncthreads();
  if (r != 0 || col >= ld) return;
  for (int i = 1; i < 16; ++i) s += sums[i][c];
  T* out = col < width ? out0 : out1;
  const int64_t at = col < width ? col : col - width;
  if (out != nullptr && at < valid) out[at] = narrow<T>(s);
}

// C = the splits' partial sums (+ bias + R), in the order of the splits.
template <class T>
__global__ __launch_bounds__(GROUP) void reduce_splits_kernel(const float* part, int splits,
                                                              GemmArgs p) {
  const int64_t per = (p.N + 3) / 4;
  const int64_t at = int64_t(blockIdx.x) * GROUP + threadIdx.x;
  const int64_t m = at / per, n = (at - m * per) * 4;
  if (m >= p.M) return;
  const int64_t row = m < p.half ? m : m - p.half;
  if (row >= p.rows) return;
  const int valid = int(min(int64_t(4), p.N - n));
  const int64_t ldp = per * 4;
  floatx4 s = *reinterpret_cast<const floatx4*>(part + m * ldp + n);
  for (int i = 1; i < splits; ++i)
    s += *reinterpret_cast<const floatx4*>(part + (i * p.M + m) * ldp + n);
  float x[4] = {s[0], s[1], s[2], s[3]}, y[4];
  if (p.bias != nullptr) {
    load_wide<4>(static_cast<const T*>(p.bias) + n, valid, y);
    for (int e = 0; e < 4; ++e) x[e] += y[e];
  }
  if (p.R != nullptr) {
    load_wide<4>(static_cast<const T*>(p.R) + m * p.ldr + n, valid, y);
    for (int e = 0; e < 4; ++e) x[e] += y[e];
  }
  T* out = static_cast<T*>(p.out[m < p.half ? 0 : 1]);
  if (out != nullptr) store_wide<4>(out + row * p.ldo + n, valid, x);
}

// Zero rows: weights' gradients are zero.
template <class T>
__global__ __launch_bounds__(GROUP) void clear_kernel(T* p, int64_t rows, int64_t cols, int64_t ld) {
  const int64_t at = int64_t(blockIdx.x) * GROUP + threadIdx.x;
  if (at < rows * cols) p[at / cols * ld + at % cols] = narrow<T>(0.f);
}

// ---------------------------------------------------------------- products

// Tiles of C.  256 x 256 by eight waves of 128 x 64, one workgroup to a CU: the
// LDS reads of a k step (96 bytes a clock at the matrix unit's full rate)
// stay below its 128; 1,150 TFLOP/s at 16384 x 2048 x 8192 against 930 of four
// waves of 128 x 128 and 840 of the 128 x 128 tile, whose 64 x 64 waves take all 128.  The smaller one
// where the larger would leave CUs without a tile.
constexpr int TILE = 128;
constexpr int BIG_TILE = 256;
constexpr int64_t CUS = 256;

// Parts of k: products with few tiles are split until two workgroups per CU
// have work, at four k tiles each or more.
int pick_splits(int64_t M, int64_t N, int64_t ktiles) {
  const int64_t tiles = std::max<int64_t>(1, ceil_div(M, TILE) * ceil_div(N, TILE));
  const int64_t want = 2 * CUS / tiles;
  return int(std::max<int64_t>(1, std::min(want, ktiles / 4)));
}
size_t split_floats(int64_t M, int64_t N, int64_t ktiles) {
  const int s = pick_splits(M, N, ktiles);
  return s == 1 ? 0 : size_t(s) * size_t(M) * size_t(round_up(N, 4));
}

void check_grid(int64_t groups) {
  FD_REQUIRE(groups < (int64_t(1) << 31), FD_ERR_UNSUPPORTED, "problem too large for one launch");
}

template <int BM, int BN, int WM, int WN, bool ACOL, bool BCOL, int EPI, class T, int ACT>
void launch_config(GemmArgs& p, hipStream_t stream) {
  constexpr int BH = EPI == GATE ? BN / 2 : BN;
  constexpr size_t lds = 2 * (BM + BN) * BK * 2;
  p.tiles_m = ceil_div(p.M, BM);
  p.tiles_n = ceil_div(p.N, BH);
  auto kernel = gemm_kernel<BM, BN, WM, WN, ACOL, BCOL, EPI, T, ACT>;
  FD_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                   hipFuncAttributeMaxDynamicSharedMemorySize, int(lds)));
  check_grid(p.tiles_m * p.tiles_n * p.splits);
  kernel<<<dim3(unsigned(p.tiles_m * p.tiles_n * p.splits)), dim3(WM * WN * WAVE), lds, stream>>>(p);
  FD_LAUNCH_CHECK();
}

bool big_tiles(int64_t M, int64_t N) {
  return ceil_div(M, BIG_TILE) * ceil_div(N, BIG_TILE) >= CUS;
}

template <bool ACOL, bool BCOL, int EPI, class T, int ACT>
void launch_tile(GemmArgs& p, hipStream_t stream) {
  if (big_tiles(p.M, EPI == GATE ? 2 * p.N : p.N))
    launch_config<BIG_TILE, BIG_TILE, 2, 4, ACOL, BCOL, EPI, T, ACT>(p, stream);
  else
    launch_config<TILE, TILE, 2, 2, ACOL, BCOL, EPI, T, ACT>(p, stream);
}

// C stored as T, through partial sums where k is split.
template <bool ACOL, bool BCOL, class T>
void launch_store(GemmArgs& p, float* part, hipStream_t stream) {
  p.splits = pick_splits(p.M, p.N, p.ktiles * p.segs);
  if (p.splits == 1) {
    launch_tile<ACOL, BCOL, STORE, T, 0>(p, stream);
    return;
  }
  GemmArgs q = p;
  q.bias = q.R = nullptr;
  q.out[0] = part;
  q.ldo = round_up(p.N, 4);
  q.half = q.rows = p.M;
  launch_tile<ACOL, BCOL, STORE, float, 0>(q, stream);
  const int64_t groups = ceil_div(p.M * ceil_div(p.N, 4), GROUP);
  check_grid(groups);
  reduce_splits_kernel<T><<<dim3(unsigned(groups)), dim3(GROUP), 0, stream>>>(part, p.splits, p);
  FD_LAUNCH_CHECK();
}

// ---------------------------------------------------------------- the block

// A matrix operand in memory: as given where the product can load it, else packed.
struct Matrix {
  const bf16* p = nullptr;
  int64_t ld = 0, rows = 0, cols = 0, plane = 0;  // cols: a multiple of 8
};

int planes_of(int type) { return type == FD_F32 ? PLANES : 1; }

struct Work {
  bf16 *x = nullptr, *wg = nullptr, *wu = nullptr, *wd = nullptr, *dy = nullptr;
  bf16 *h = nullptr, *dgu = nullptr;
  float *part = nullptr, *colsum = nullptr, *saved = nullptr;
  PackJobs jobs;
};

int64_t f_padded(int64_t F) { return round_up(F, BK); }

size_t packed(int64_t rows, int64_t cols, int type) {
  return size_t(rows) * size_t(round_up(cols, 8)) * planes_of(type);
}
// k tiles of the contraction over n, and stretches of one matrix pair
int segs_of(int type) { return type == FD_F32 ? PAIRS : 1; }

constexpr int64_t SUM_ROWS = 64;  // row groups of dY's column sums
size_t saved_floats(int64_t N, int64_t F) { return size_t(round_up(N, 32)) * f_padded(F) * 2; }

Work carve_work(Arena& a, const fd_gated_block& b, int backward) {
  Work w;
  const int t = b.type, s = segs_of(t);
  w.x = a.take<bf16>(packed(b.N, b.D, t));
  w.wg = a.take<bf16>(packed(b.F, b.D, t));
  w.wu = a.take<bf16>(packed(b.F, b.D, t));
  w.wd = a.take<bf16>(packed(b.O, b.F, t));
  const int64_t Fp = f_padded(b.F);
  w.h = a.take<bf16>(size_t(b.N) * Fp * planes_of(t));
  size_t part = 0;
  if (backward == 0) {
    part = split_floats(b.N, b.O, Fp / BK * s);
  } else {
    w.dy = a.take<bf16>(packed(b.N, b.O, t));
    w.dgu = a.take<bf16>(size_t(b.N) * 2 * Fp * planes_of(t));
    w.colsum = a.take<float>(std::max(size_t(ceil_div(b.N, TILE)) * 2 * 2 * Fp,
                                      size_t(SUM_ROWS) * size_t(b.O)));
    const int64_t nt = ceil_div(b.N, BK) * s;
    part = std::max({split_floats(b.N, b.D, 2 * Fp / BK * s), split_floats(2 * Fp, b.D, nt),
                     split_floats(b.O, b.F, nt)});
    if (backward == 2) w.saved = a.take<float>(saved_floats(b.N, b.F));
  }
  w.part = a.take<float>(part);
  return w;
}

bool direct(const void* p, int64_t ld, int64_t cols, int type) {
  return type == FD_BF16 && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 &&
         cols % 8 == 0 && ld < MAX_LD;
}

Matrix bring(Work& w, const void* p, int64_t ld, int64_t rows, int64_t cols, int type, bf16* room) {
  if (direct(p, ld, cols, type)) return Matrix{static_cast<const bf16*>(p), ld, rows, cols, 0};
  const int64_t ldp = round_up(cols, 8);
  PackJob& j = w.jobs.j[w.jobs.count++];
  j = PackJob{p, ld, rows, cols, ldp, room, rows * ldp, w.jobs.groups};
  w.jobs.groups += ceil_div(rows * (ldp / 8), GROUP);
  return Matrix{room, ldp, rows, ldp, rows * ldp};
}

void run_pack(const PackJobs& jobs, int type, hipStream_t stream) {
  if (jobs.count == 0) return;
  check_grid(jobs.groups);
  if (type == FD_F32)
    pack_kernel<float><<<dim3(unsigned(jobs.groups)), dim3(GROUP), 0, stream>>>(jobs);
  else
    pack_kernel<bf16><<<dim3(unsigned(jobs.groups)), dim3(GROUP), 0, stream>>>(jobs);
  FD_LAUNCH_CHECK();
}

// The plane pairs of x y that reach 2^-24 of it, smallest first.
constexpr int PAIR_A[PAIRS] = {1, 0, 2, 0, 1, 0};
constexpr int PAIR_B[PAIRS] = {1, 2, 0, 1, 0, 0};

// Stretches of matrix `which` (0 or 1 of those contracted one after the other).
void set_rows(Operand& o, const Matrix& m, int type, int which, bool is_a, int64_t extent) {
  const int s = segs_of(type);
  for (int i = 0; i < s; ++i)
    o.p[which * s + i] = m.p + (type == FD_F32 ? (is_a ? PAIR_A : PAIR_B)[i] * m.plane : 0);
  o.ld = m.ld;
  o.rows = extent;
}

Matrix view_h(const Work& w, const fd_gated_block& b) {
  const int64_t Fp = f_padded(b.F);
  return Matrix{w.h, Fp, b.N, Fp, b.N * Fp};
}

template <class T>
void by_act(const fd_gated_block& b, GemmArgs& p, int epi, hipStream_t st) {
  p.splits = 1;
  if (epi == GATE) {
    if (b.act == FD_ACT_SILU) launch_tile<false, false, GATE, T, FD_ACT_SILU>(p, st);
    else launch_tile<false, false, GATE, T, FD_ACT_GELU>(p, st);
  } else {
    if (b.act == FD_ACT_SILU) launch_tile<false, true, GRAD, T, FD_ACT_SILU>(p, st);
    else launch_tile<false, true, GRAD, T, FD_ACT_GELU>(p, st);
  }
}

// G, U (kept where `saved`) and H (where `h`).
template <class T>
void run_gate(const fd_gated_block& b, const Work& w, const Matrix& x, const Matrix& wg,
              const Matrix& wu, float* saved, bool h, hipStream_t st) {
  GemmArgs p{};
  p.M = b.N;
  p.N = b.F;
  p.segs = segs_of(b.type);
  p.ktiles = ceil_div(x.cols, BK);
  set_rows(p.a, x, b.type, 0, true, b.N);
  set_rows(p.b, wg, b.type, 0, false, b.F);
  set_rows(p.b2, wu, b.type, 0, false, b.F);
  p.a.k = p.b.k = p.b2.k = x.cols;
  p.bg = b.bg;
  p.bu = b.bu;
  p.saved = saved;
  p.Fp = f_padded(b.F);
  p.H = h ? w.h : nullptr;
  p.hplane = b.N * p.Fp;
  by_act<T>(b, p, GATE, st);
}

void check_block(const fd_gated_block* bp) {
  FD_REQUIRE(bp != nullptr, FD_ERR_INVALID_ARG, "block is NULL");
  const fd_gated_block& b = *bp;
  check_dtype(b.type, "dtype");
  FD_REQUIRE(b.N >= 0 && b.N <= MAX_ROWS, FD_ERR_INVALID_ARG, "N out of range [0, 2^30]");
  FD_REQUIRE(b.D >= 1 && b.F >= 1 && b.O >= 1, FD_ERR_INVALID_ARG, "widths must be >= 1");
  FD_REQUIRE(b.D <= MAX_WIDTH && b.F <= MAX_WIDTH && b.O <= MAX_WIDTH, FD_ERR_UNSUPPORTED,
             "widths above 2^20 are not supported");
}

void check_arrays(const fd_gated_block& b) {
  FD_REQUIRE(b.act == FD_ACT_SILU || b.act == FD_ACT_GELU, FD_ERR_INVALID_ARG,
             "unknown activation");
  FD_REQUIRE(b.Wg != nullptr && b.Wu != nullptr && b.Wd != nullptr, FD_ERR_INVALID_ARG,
             "a weight is NULL");
  FD_REQUIRE(b.N == 0 || b.X != nullptr, FD_ERR_INVALID_ARG, "X is NULL");
  FD_REQUIRE(b.ldx >= b.D && b.ldwi >= b.D && b.ldwd >= b.F, FD_ERR_INVALID_ARG,
             "leading dimensions must cover the rows");
  for (const void* p : {b.X, b.Wg, b.Wu, b.Wd, b.bg, b.bu, b.bd})
    check_element_aligned(p, b.type, "an array of the block");
}

void check_saved(const fd_gated_block& b, const void* saved, size_t bytes) {
  if (saved == nullptr) return;
  FD_REQUIRE(bytes >= saved_floats(b.N, b.F) * sizeof(float), FD_ERR_WORKSPACE,
             "saved is too small");
  FD_REQUIRE((reinterpret_cast<uintptr_t>(saved) & 255) == 0, FD_ERR_WORKSPACE,
             "saved must be 256-byte aligned");
}

Work carve_checked(const fd_gated_block& b, int backward, void* ws, size_t ws_bytes) {
  Arena m;
  m.measuring = true;
  carve_work(m, b, backward);
  check_workspace(ws, ws_bytes, m.used);
  Arena a;
  a.base = static_cast<char*>(ws);
  a.cap = ws_bytes;
  return carve_work(a, b, backward);
}

template <class T>
void forward(const fd_gated_block& b, Work& w, const void* R, int64_t ldr, void* Y, int64_t ldy,
             float* saved, hipStream_t st) {
  const int t = b.type;
  const Matrix x = bring(w, b.X, b.ldx, b.N, b.D, t, w.x);
  const Matrix wg = bring(w, b.Wg, b.ldwi, b.F, b.D, t, w.wg);
  const Matrix wu = bring(w, b.Wu, b.ldwi, b.F, b.D, t, w.wu);
  const Matrix wd = bring(w, b.Wd, b.ldwd, b.O, b.F, t, w.wd);
  run_pack(w.jobs, t, st);
  run_gate<T>(b, w, x, wg, wu, saved, true, st);
  GemmArgs p{};
  const Matrix h = view_h(w, b);
  p.M = b.N;
  p.N = b.O;
  p.segs = segs_of(t);
  p.ktiles = h.cols / BK;
  set_rows(p.a, h, t, 0, true, b.N);
  set_rows(p.b, wd, t, 0, false, b.O);
  p.a.k = h.cols;
  p.b.k = wd.cols;
  p.out[0] = Y;
  p.ldo = ldy;
  p.half = p.rows = b.N;
  p.bias = b.bd;
  p.R = R;
  p.ldr = ldr;
  launch_store<false, false, T>(p, w.part, st);
}

template <class T>
void clear(void* p, int64_t rows, int64_t cols, int64_t ld, hipStream_t st) {
  if (p == nullptr) return;
  const int64_t groups = ceil_div(rows * cols, GROUP);
  check_grid(groups);
  clear_kernel<T><<<dim3(unsigned(groups)), dim3(GROUP), 0, st>>>(static_cast<T*>(p), rows, cols, ld);
  FD_LAUNCH_CHECK();
}

template <class T>
void backward(const fd_gated_block& b, Work& w, const void* dY, int64_t lddy, const float* saved,
              const fd_gated_grads& g, hipStream_t st) {
  const int t = b.type;
  if (b.N == 0) {
    clear<T>(g.dWg, b.F, b.D, g.lddwi, st);
    clear<T>(g.dWu, b.F, b.D, g.lddwi, st);
    clear<T>(g.dWd, b.O, b.F, g.lddwd, st);
    clear<T>(g.dbg, 1, b.F, b.F, st);
    clear<T>(g.dbu, 1, b.F, b.F, st);
    clear<T>(g.dbd, 1, b.O, b.O, st);
    return;
  }
  const bool inner = g.dX != nullptr || g.dWg != nullptr || g.dWu != nullptr ||
                     g.dbg != nullptr || g.dbu != nullptr || g.dWd != nullptr;
  const int64_t Fp = f_padded(b.F);
  if (inner) {
    const bool gate = saved == nullptr;
    const bool need_x = gate || g.dWg != nullptr || g.dWu != nullptr;
    const bool need_w = gate || g.dX != nullptr;
    Matrix x, wg, wu;
    if (need_x) x = bring(w, b.X, b.ldx, b.N, b.D, t, w.x);
    if (need_w) {
      wg = bring(w, b.Wg, b.ldwi, b.F, b.D, t, w.wg);
      wu = bring(w, b.Wu, b.ldwi, b.F, b.D, t, w.wu);
    }
    const Matrix wd = bring(w, b.Wd, b.ldwd, b.O, b.F, t, w.wd);
    const Matrix dy = bring(w, dY, lddy, b.N, b.O, t, w.dy);
    run_pack(w.jobs, t, st);
    if (gate) {
      run_gate<T>(b, w, x, wg, wu, w.saved, false, st);
      saved = w.saved;
    }
    {  // dH, and from it dG, dU, H
      GemmArgs p{};
      p.M = b.N;
      p.N = b.F;
      p.segs = segs_of(t);
      p.ktiles = ceil_div(b.O, BK);
      set_rows(p.a, dy, t, 0, true, b.N);
      set_rows(p.b, wd, t, 0, false, wd.cols);
      p.a.k = dy.cols;
      p.b.k = b.O;
      p.saved = const_cast<float*>(saved);
      p.Fp = Fp;
      p.H = w.h;
      p.hplane = b.N * Fp;
      p.dGU = w.dgu;
      p.gplane = b.N * 2 * Fp;
      p.colsum = g.dbg != nullptr || g.dbu != nullptr ? w.colsum : nullptr;
      by_act<T>(b, p, GRAD, st);
      if (p.colsum != nullptr) {
        reduce_columns_kernel<T><<<dim3(unsigned(ceil_div(2 * Fp, 16))), dim3(GROUP), 0, st>>>(
            w.colsum, p.tiles_m * 2, 2 * Fp, Fp, b.F, static_cast<T*>(g.dbg),
            static_cast<T*>(g.dbu));
        FD_LAUNCH_CHECK();
      }
    }
    const Matrix h = view_h(w, b);
    const Matrix dgu{w.dgu, 2 * Fp, b.N, 2 * Fp, b.N * 2 * Fp};
    const Matrix du{w.dgu + Fp, 2 * Fp, b.N, Fp, b.N * 2 * Fp};
    if (g.dX != nullptr) {  // [dG dU] [Wg; Wu]
      GemmArgs p{};
      p.M = b.N;
      p.N = b.D;
      p.segs = 2 * segs_of(t);
      p.ktiles = Fp / BK;
      set_rows(p.a, dgu, t, 0, true, b.N);
      set_rows(p.a, du, t, 1, true, b.N);
      set_rows(p.b, wg, t, 0, false, wg.cols);
      set_rows(p.b, wu, t, 1, false, wu.cols);
      p.a.k = Fp;
      p.b.k = b.F;
      p.out[0] = g.dX;
      p.ldo = g.lddx;
      p.half = p.rows = b.N;
      launch_store<false, true, T>(p, w.part, st);
    }
    if (g.dWg != nullptr || g.dWu != nullptr) {  // [dG dU]^T X
      GemmArgs p{};
      p.M = 2 * Fp;
      p.N = b.D;
      p.segs = segs_of(t);
      p.ktiles = ceil_div(b.N, BK);
      set_rows(p.a, dgu, t, 0, true, 2 * Fp);
      set_rows(p.b, x, t, 0, false, x.cols);
      p.a.k = p.b.k = b.N;
      p.out[0] = g.dWg;
      p.out[1] = g.dWu;
      p.ldo = g.lddwi;
      p.half = Fp;
      p.rows = b.F;
      launch_store<true, true, T>(p, w.part, st);
    }
    if (g.dWd != nullptr) {  // dY^T H
      GemmArgs p{};
      p.M = b.O;
      p.N = b.F;
      p.segs = segs_of(t);
      p.ktiles = ceil_div(b.N, BK);
      set_rows(p.a, dy, t, 0, true, dy.cols);
      set_rows(p.b, h, t, 0, false, h.cols);
      p.a.k = p.b.k = b.N;
      p.out[0] = g.dWd;
      p.ldo = g.lddwd;
      p.half = p.rows = b.O;
      launch_store<true, true, T>(p, w.part, st);
    }
  }
  if (g.dbd != nullptr) {
    const int64_t rows = std::min<int64_t>(SUM_ROWS, ceil_div(b.N, 4));
    column_sum_kernel<T><<<dim3(unsigned(ceil_div(b.O, WAVE)), unsigned(rows)), dim3(GROUP), 0, st>>>(
        static_cast<const T*>(dY), lddy, b.N, b.O, w.colsum);
    FD_LAUNCH_CHECK();
    reduce_columns_kernel<T><<<dim3(unsigned(ceil_div(b.O, 16))), dim3(GROUP), 0, st>>>(
        w.colsum, rows, b.O, b.O, b.O, static_cast<T*>(g.dbd), nullptr);
    FD_LAUNCH_CHECK();
  }
}

}  // namespace
}  // namespace net
}  // namespace fd

using namespace fd;
using namespace fd::net;

extern "C" {

size_t fd_gated_saved_size(const fd_gated_block* b) {
  size_t out = 0;
  const fd_status st = guarded([&] {
    check_block(b);
    out = saved_floats(b->N, b->F) * sizeof(float);
  });
  return st == FD_OK ? out : 0;
}

size_t fd_gated_workspace_size(const fd_gated_block* b, int32_t backward) {
  size_t out = 0;
  const fd_status st = guarded([&] {
    check_block(b);
    FD_REQUIRE(backward >= 0 && backward <= 2, FD_ERR_INVALID_ARG, "backward must be 0, 1 or 2");
    Arena a;
    a.measuring = true;
    carve_work(a, *b, backward);
    out = a.used;
  });
  return st == FD_OK ? out : 0;
}

fd_status fd_gated_forward(const fd_gated_block* b, const void* R, int64_t ldr, void* Y,
                           int64_t ldy, void* saved, size_t saved_bytes, void* ws,
                           size_t ws_bytes, void* stream) {
  return guarded([&] {
    check_block(b);
    check_arrays(*b);
    FD_REQUIRE(b->N == 0 || Y != nullptr, FD_ERR_INVALID_ARG, "Y is NULL");
    FD_REQUIRE(ldy >= b->O && (R == nullptr || ldr >= b->O), FD_ERR_INVALID_ARG,
               "leading dimensions must cover the rows");
    FD_REQUIRE(R != Y || b->N == 0 || ldr == ldy, FD_ERR_INVALID_ARG, "Y = R needs ldy = ldr");
    check_element_aligned(R, b->type, "R");
    check_element_aligned(Y, b->type, "Y");
    check_saved(*b, saved, saved_bytes);
    if (b->N == 0) return;
    Work w = carve_checked(*b, 0, ws, ws_bytes);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (b->type == FD_F32)
      forward<float>(*b, w, R, ldr, Y, ldy, static_cast<float*>(saved), st);
    else
      forward<bf16>(*b, w, R, ldr, Y, ldy, static_cast<float*>(saved), st);
  });
}

fd_status fd_gated_backward(const fd_gated_block* b, const void* dY, int64_t lddy,
                            const void* saved, size_t saved_bytes, const fd_gated_grads* grads,
                            void* ws, size_t ws_bytes, void* stream) {
  return guarded([&] {
    check_block(b);
    check_arrays(*b);
    FD_REQUIRE(grads != nullptr, FD_ERR_INVALID_ARG, "grads is NULL");
    const fd_gated_grads& g = *grads;
    FD_REQUIRE(b->N == 0 || dY != nullptr, FD_ERR_INVALID_ARG, "dY is NULL");
    FD_REQUIRE(lddy >= b->O, FD_ERR_INVALID_ARG, "lddy must be >= O");
    FD_REQUIRE((g.dX == nullptr || g.lddx >= b->D) &&
                   ((g.dWg == nullptr && g.dWu == nullptr) || g.lddwi >= b->D) &&
                   (g.dWd == nullptr || g.lddwd >= b->F),
               FD_ERR_INVALID_ARG, "leading dimensions of the gradients must cover the rows");
    check_element_aligned(dY, b->type, "dY");
    for (const void* p : {g.dX, g.dWg, g.dWu, g.dWd, g.dbg, g.dbu, g.dbd})
      check_element_aligned(p, b->type, "a gradient");
    check_saved(*b, saved, saved_bytes);
    Work w;
    if (b->N > 0) w = carve_checked(*b, saved == nullptr ? 2 : 1, ws, ws_bytes);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (b->type == FD_F32)
      backward<float>(*b, w, dY, lddy, static_cast<const float*>(saved), g, st);
    else
      backward<bf16>(*b, w, dY, lddy, static_cast<const float*>(saved), g, st);
  });
}

}  // extern "C"
