// The gated feed-forward block, forward and backward.
#include <algorithm>
#include <cmath>

#include "fd_guard.hpp"
#include "fd_solver.hpp"
#include "net_gemm.hpp"
#include "net_narrow.hpp"
#include "net_skinny.hpp"

namespace fd {
namespace net {
namespace {

constexpr int GROUP = 256;

// ---------------------------------------------------------------- before
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
// Up to five matrices to pack, then the partial column sums of one (dY):
// workgroup y of `parts` adds its stretch of rows.
constexpr int PACK_JOBS = 5;
struct PackJobs {
  PackJob j[PACK_JOBS];
  int count = 0;
  int64_t groups = 0;
  const void* sum = nullptr;
  int64_t sum_ld, sum_rows, sum_cols, sum_parts;
  float* sum_out;
};

template <class T>
__device__ void column_sums(const PackJobs& jobs, int64_t id) {
  __shared__ float sums[4][WAVE];
  const int64_t cols = jobs.sum_cols, across = (cols + WAVE - 1) / WAVE;
  const int64_t y = id / across, col = (id - y * across) * WAVE + threadIdx.x % WAVE;
  const int r = threadIdx.x / WAVE;
  const int64_t r0 = jobs.sum_rows * y / jobs.sum_parts, r1 = jobs.sum_rows * (y + 1) / jobs.sum_parts;
  float s = 0.f;
  if (col < cols) {
    const T* p = static_cast<const T*>(jobs.sum) + col;
    int64_t i = r0 + r;
    for (; i + 12 < r1; i += 16) {
      const float a = widen(p[i * jobs.sum_ld]), b = widen(p[(i + 4) * jobs.sum_ld]);
      const float c = widen(p[(i + 8) * jobs.sum_ld]), d = widen(p[(i + 12) * jobs.sum_ld]);
      s += (a + b) + (c + d);
    }
    for (; i < r1; i += 4) s += widen(p[i * jobs.sum_ld]);
  }
  sums[r][threadIdx.x % WAVE] = s;
  __syncthreads();
  if (r == 0 && col < cols) {
    for (int i = 1; i < 4; ++i) s += sums[i][threadIdx.x];
    jobs.sum_out[y * cols + col] = s;
  }
}

template <class T>
__global__ __launch_bounds__(GROUP) void before_kernel(PackJobs jobs, int64_t first) {
  const int64_t id = first + blockIdx.x;
  if (id >= jobs.groups) {
    column_sums<T>(jobs, id - jobs.groups);
    return;
  }
  int i = 0;
  while (i + 1 < jobs.count && jobs.j[i + 1].first <= id) ++i;
  const PackJob& job = jobs.j[i];
  const int64_t at = (id - job.first) * GROUP + threadIdx.x;
  const int64_t per = job.ldp / 8, row = at / per, col = (at - row * per) * 8;
  if (row >= job.rows) return;
  float x[8];
  load_wide<8>(static_cast<const T*>(job.src) + row * job.ld + col,
               int(min(int64_t(8), job.cols - col)), x);
  write_planes<planes_of<T>>(job.dst + row * job.ldp + col, job.plane, x);
}

// ---------------------------------------------------------------- after
// What is left once the products are done: the sums over the parts of split
// contractions, and over partial column sums; each in one fixed order.
struct SplitJob {
  const float* part;
  int splits;
  int64_t M, N, ldp;
  void* out[2];
  int64_t ldo, half, rows;
  const void *bias, *R;
  int64_t ldr;
  int64_t first;
};
struct ColumnJob {  // column c of the first `valid` of every `width` goes to out[c / width]
  const float* part;
  int64_t rows, ld, width, valid;
  void* out[2];
  int64_t first;
};
struct AfterJobs {
  SplitJob s[GROUP_GEMMS];
  ColumnJob c[2];
  int splits = 0, columns = 0;
  int64_t groups = 0;
};

// C = the parts (+ bias + R): four columns of a row a thread.
template <class T>
__device__ void sum_splits(const SplitJob& p, int64_t id) {
  const int64_t per = (p.N + 3) / 4;
  const int64_t at = id * GROUP + threadIdx.x;
  const int64_t m = at / per, n = (at - m * per) * 4;
  if (m >= p.M) return;
  const int64_t row = m < p.half ? m : m - p.half;
  T* out = static_cast<T*>(p.out[m < p.half ? 0 : 1]);
  if (row >= p.rows || out == nullptr) return;
  const int valid = int(min(int64_t(4), p.N - n));
  const floatx4* q = reinterpret_cast<const floatx4*>(p.part + m * p.ldp + n);
  const int64_t step = p.M * p.ldp / 4;
  floatx4 s = {0.f, 0.f, 0.f, 0.f};
  int i = 0;
  for (; i + 4 <= p.splits; i += 4) {
    const floatx4 a = q[i * step], b = q[(i + 1) * step], c = q[(i + 2) * step],
                  d = q[(i + 3) * step];
    s += (a + b) + (c + d);
  }
  for (; i < p.splits; ++i) s += q[i * step];
  float x[4] = {s[0], s[1], s[2], s[3]}, y[4];
  if (p.bias != nullptr) {
    load_wide<4>(static_cast<const T*>(p.bias) + n, valid, y);
    for (int e = 0; e < 4; ++e) x[e] += y[e];
  }
  if (p.R != nullptr) {
    load_wide<4>(static_cast<const T*>(p.R) + m * p.ldr + n, valid, y);
    for (int e = 0; e < 4; ++e) x[e] += y[e];
  }
  store_wide<4>(out + row * p.ldo + n, valid, x);
}

// Sixteen columns a workgroup, sixteen rows at a time.
template <class T>
__device__ void sum_columns(const ColumnJob& p, int64_t id) {
  __shared__ float sums[16][17];
  const int c = threadIdx.x % 16, r = threadIdx.x / 16;
  const int64_t col = id * 16 + c;
  float s = 0.f;
  if (col < p.ld)
    for (int64_t i = r; i < p.rows; i += 16) s += p.part[i * p.ld + col];
  sums[r][c] = s;
  __syncthreads();
  if (r != 0 || col >= p.ld) return;
  for (int i = 1; i < 16; ++i) s += sums[i][c];
  T* out = static_cast<T*>(p.out[col < p.width ? 0 : 1]);
  const int64_t at = col < p.width ? col : col - p.width;
  if (out != nullptr && at < p.valid) out[at] = narrow<T>(s);
}

template <class T>
__global__ __launch_bounds__(GROUP) void after_kernel(AfterJobs jobs) {
  const int64_t id = blockIdx.x;
  for (int i = jobs.columns - 1; i >= 0; --i)
    if (id >= jobs.c[i].first) return sum_columns<T>(jobs.c[i], id - jobs.c[i].first);
  int i = 0;
  while (i + 1 < jobs.splits && jobs.s[i + 1].first <= id) ++i;
  sum_splits<T>(jobs.s[i], id - jobs.s[i].first);
}

// Zero rows: weights' gradients are zero.
template <class T>
__global__ __launch_bounds__(GROUP) void clear_kernel(T* p, int64_t rows, int64_t cols, int64_t ld) {
  for (int64_t at = int64_t(blockIdx.x) * GROUP + threadIdx.x; at < rows * cols;
       at += int64_t(gridDim.x) * GROUP)
    p[at / cols * ld + at % cols] = narrow<T>(0.f);
}

// ---------------------------------------------------------------- products

template <int C, int EPI, class T>
struct Config;  // BM, BN, WM, WN
template <int EPI, class T>
struct Config<BIG, EPI, T> {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int bm = 256, bn = F32 ? 128 : 256, wm = F32 ? 4 : 2, wn = F32 ? 2 : 4;
};
template <int EPI, class T>
struct Config<MID, EPI, T> {
  static constexpr int bm = 128, bn = 128, wm = 2, wn = 2;
};
template <int EPI, class T>
struct Config<SMALL, EPI, T> {
  static constexpr int bm = 64, bn = 64, wm = 2, wn = EPI == GATE ? 1 : 2;
};

template <class K>
void allow_lds(K kernel, size_t bytes) {
  FD_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                   hipFuncAttributeMaxDynamicSharedMemorySize, int(bytes)));
}

template <int C, bool ACOL, bool BCOL, int EPI, class T, int ACT, int HP>
void launch_config(GemmArgs& p, hipStream_t stream) {
  using K = Config<C, EPI, T>;
  constexpr int PL = planes_of<T>, PLA = EPI == STORE ? HP : PL;
  constexpr size_t lds = gemm_lds<K::bm, K::bn, T, PLA, PL>;
  p.tiles_m = ceil_div(p.M, K::bm);
  // GATE and GRAD write whole padded rows
  p.tiles_n = ceil_div(EPI == STORE ? p.N : p.Fp, EPI == GATE ? K::bn / 2 : K::bn);
  const int64_t groups = p.tiles_m * p.tiles_n * p.splits;
  constexpr int THREADS = K::wm * K::wn * WAVE;
  check_launch(groups, THREADS);
  auto kernel = gemm_kernel<K::bm, K::bn, K::wm, K::wn, ACOL, BCOL, EPI, T, ACT, PLA, PL, HP>;
  allow_lds(kernel, lds);
  kernel<<<dim3(unsigned(groups)), dim3(THREADS), lds, stream>>>(p);
  FD_LAUNCH_CHECK();
}

template <bool ACOL, bool BCOL, int EPI, class T, int ACT, int HP>
void launch(int config, GemmArgs& p, hipStream_t stream) {
  if constexpr (HP == planes_of<T>) {
    if (config == BIG) return launch_config<BIG, ACOL, BCOL, EPI, T, ACT, HP>(p, stream);
    if (config == MID) return launch_config<MID, ACOL, BCOL, EPI, T, ACT, HP>(p, stream);
  }
  launch_config<SMALL, ACOL, BCOL, EPI, T, ACT, HP>(p, stream);
}

// GATE or GRAD in the tile and parts of a plan, and the rest where there are parts.
template <bool BCOL, int EPI, class T, int ACT, int HP>
void launch_inner(int config, const Shape& s, float* part, GemmArgs& p, hipStream_t stream) {
  p.splits = s.splits;
  p.part = part;
  launch<false, BCOL, EPI, T, ACT, HP>(config, p, stream);
  if (s.splits == 1) return;
  const int64_t groups = ceil_div(ceil_div(p.M, 32) * (p.Fp / 32), GROUP / WAVE);
  check_launch(groups, GROUP);
  finish_kernel<EPI, T, ACT, HP><<<dim3(unsigned(groups)), dim3(GROUP), 0, stream>>>(p);
  FD_LAUNCH_CHECK();
}

template <int C, class T, int HP>
void launch_group(GemmGroup& s, hipStream_t stream) {
  using K = Config<C, STORE, T>;
  constexpr size_t lds = gemm_lds<K::bm, K::bn, T, HP, planes_of<T>>;
  static_assert(K::bm == K::bn || HP == planes_of<T>, "the same LDS for planes of a and of b");
  int64_t at = 0;
  for (int i = 0; i < s.count; ++i) {
    GemmArgs& p = s.g[i];
    p.tiles_m = ceil_div(p.M, K::bm);
    p.tiles_n = ceil_div(p.N, K::bn);
    s.first[i] = at;
    at += p.tiles_m * p.tiles_n * p.splits;
  }
  s.first[s.count] = at;
  constexpr int THREADS = K::wm * K::wn * WAVE;
  check_launch(at, THREADS);
  auto kernel = gemm_group_kernel<K::bm, K::bn, K::wm, K::wn, T, HP>;
  allow_lds(kernel, lds);
  kernel<<<dim3(unsigned(at)), dim3(THREADS), lds, stream>>>(s);
  FD_LAUNCH_CHECK();
}

// A split product's parts, and their sum after it.
void set_parts(GemmArgs& p, const Shape& s, float*& room, AfterJobs& after) {
  p.splits = s.splits;
  if (s.splits == 1) return;
  p.part = room;
  p.ldp = round_up(p.N, 4);
  room += s.part();
  SplitJob& j = after.s[after.splits++];
  j = SplitJob{p.part, s.splits, p.M, p.N, p.ldp, {p.out[0], p.out[1]}, p.ldo, p.half, p.rows,
               p.bias, p.R, p.ldr, after.groups};
  after.groups += ceil_div(p.M * ceil_div(p.N, 4), GROUP);
}
void add_columns(AfterJobs& after, const float* part, int64_t rows, int64_t ld, int64_t width,
                 int64_t valid, void* out0, void* out1) {
  after.c[after.columns++] = ColumnJob{part, rows, ld, width, valid, {out0, out1}, after.groups};
  after.groups += ceil_div(ld, 16);
}
template <class T>
void run_after(const AfterJobs& after, hipStream_t stream) {
  if (after.groups == 0) return;
  check_launch(after.groups, GROUP);
  after_kernel<T><<<dim3(unsigned(after.groups)), dim3(GROUP), 0, stream>>>(after);
  FD_LAUNCH_CHECK();
}

// ---------------------------------------------------------------- the block

struct Work {
  bf16 *x = nullptr, *wg = nullptr, *wu = nullptr, *wd = nullptr, *dy = nullptr;
  bf16 *h = nullptr, *dgu = nullptr;
  float *part = nullptr, *colsum = nullptr, *dysum = nullptr;
  char* saved = nullptr;
  PackJobs jobs;
  GatedPlan plan;
};

template <class T>
size_t packed(int64_t rows, int64_t cols) {
  return size_t(rows) * size_t(round_up(cols, 8)) * planes_of<T>;
}

constexpr int64_t SUM_PARTS = 128;  // partial column sums of dY

template <class T>
size_t saved_bytes_t(int64_t N, int64_t F) {
  return size_t(ceil_div(N, 32)) * size_t(f_padded(F) / 32) * saved_block_bytes<T>;
}
size_t saved_bytes(const fd_gated_block& b) {
  return b.type == FD_F32 ? saved_bytes_t<float>(b.N, b.F) : saved_bytes_t<bf16>(b.N, b.F);
}

// Planes of H, dG and dU.  One bfloat16 plane rounds them once more than 32-bit
// sums would, which adds as much error to Y and to the gradients as their own
// last rounding (0.0024 from the float64 values and not 0.0017).  Where the products
// are not what takes the time, what was rounded off is a second plane: 19 -> 19.4 us at
// 2 x 32 -> 32 -> 28 (forward and backward), 29 -> 30 at 64 x 128 -> 256 -> 128,
// 31 -> 33 at 256 x 128 -> 512 -> 128; but 42 -> 52 at 1,024 x 256 -> 512 -> 256, and 147
// -> 232 at 5,003 x 509 -> 1365 -> 509, which keep one unless the caller asks for two (4.6 ->
// 14.8 ms at 16,384 x 2048 -> 8192 -> 2048: two planes take the smallest tiles alone).
constexpr double FINE_WORK = double(1 << 25);
bool fine(const fd_gated_block& b) {
  if (b.type != FD_BF16) return false;
  return (b.act & FD_GATED_FINE) != 0 ||
         double(b.N) * double(b.F) * double(std::max(b.D, b.O)) <= FINE_WORK;
}
int activation_of(const fd_gated_block& b) { return b.act & ~FD_GATED_FINE; }

template <class T>
Work carve_work_t(Arena& a, const fd_gated_block& b, int backward) {
  Work w;
  w.x = a.take<bf16>(packed<T>(b.N, b.D));
  w.wg = a.take<bf16>(packed<T>(b.F, b.D));
  w.wu = a.take<bf16>(packed<T>(b.F, b.D));
  w.wd = a.take<bf16>(packed<T>(b.O, b.F));
  const int64_t Fp = f_padded(b.F);
  const size_t blocks = size_t(ceil_div(b.N, 32)) * size_t(Fp / 32);
  const bool two = fine(b);
  const int inner = two ? 2 : planes_of<T>;
  w.h = a.take<bf16>(size_t(b.N) * Fp * inner);  // (few rows of float32: as they are)
  w.plan = plan_gated(b.N, b.D, b.F, b.O, sizeof(T) == 4, two, backward);
  const GatedPlan& p = w.plan;
  size_t part = p.gate.splits > 1 ? size_t(p.gate.splits) * blocks * 2048 : 0;
  if (backward == 0) {
    part = std::max(part, p.out[0].part());
    if (b.D <= NARROW && b.O <= NARROW)
      part = std::max(part, size_t(narrow_parts(b.N, b.F)) * size_t(b.N) * size_t(round_up(b.O, 4)));
  } else {
    w.dy = a.take<bf16>(packed<T>(b.N, b.O));
    w.dgu = a.take<bf16>(size_t(b.N) * 2 * Fp * inner);
    // a row for each 32 rows, or each row of waves of a tile: tiles of 64 or 128
    // rows have two, of 256 rows at most four
    w.colsum = a.take<float>(size_t(2 * ceil_div(b.N, 64) + 2) * 2 * Fp);
    w.dysum = a.take<float>(size_t(SUM_PARTS) * size_t(b.O));
    size_t sum = 0;
    for (const Shape& s : p.out) sum += s.part();
    part = std::max({part, sum, p.grad.splits > 1 ? size_t(p.grad.splits) * blocks * 1024 : 0});
    if (backward == 2) w.saved = a.take<char>(saved_bytes(b));
  }
  w.part = a.take<float>(part);
  return w;
}
Work carve_work(Arena& a, const fd_gated_block& b, int backward) {
  return b.type == FD_F32 ? carve_work_t<float>(a, b, backward) : carve_work_t<bf16>(a, b, backward);
}

// A matrix operand in memory: as given where the product can load it, else packed.
struct Matrix {
  const bf16* p = nullptr;
  int64_t ld = 0, rows = 0, cols = 0, plane = 0;  // cols: a multiple of 8
};

bool direct(const void* p, int64_t ld, int64_t cols, int type) {
  return type == FD_BF16 && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 &&
         cols % 8 == 0 && ld < MAX_LD;
}

Matrix pack(Work& w, const void* p, int64_t ld, int64_t rows, int64_t cols, bf16* room) {
  const int64_t ldp = round_up(cols, 8);
  PackJob& j = w.jobs.j[w.jobs.count++];
  j = PackJob{p, ld, rows, cols, ldp, room, rows * ldp, w.jobs.groups};
  w.jobs.groups += ceil_div(rows * (ldp / 8), GROUP);
  return Matrix{room, ldp, rows, ldp, rows * ldp};
}
Matrix bring(Work& w, const void* p, int64_t ld, int64_t rows, int64_t cols, int type, bf16* room) {
  if (direct(p, ld, cols, type)) return Matrix{static_cast<const bf16*>(p), ld, rows, cols, 0};
  return pack(w, p, ld, rows, cols, room);
}

template <class T>
void run_before(const PackJobs& jobs, hipStream_t stream) {
  const int64_t sums = jobs.sum == nullptr ? 0 : ceil_div(jobs.sum_cols, WAVE) * jobs.sum_parts;
  const int64_t groups = jobs.groups + sums;
  if (groups == 0) return;
  // half a launch's threads at a time: packs of 2^35 elements and more fit the memory
  constexpr int64_t SLICE = (int64_t(1) << 31) / GROUP;
  for (int64_t first = 0; first < groups; first += SLICE) {
    before_kernel<T><<<dim3(unsigned(std::min(SLICE, groups - first))), dim3(GROUP), 0, stream>>>(jobs, first);
    FD_LAUNCH_CHECK();
  }
}

// Operand rows (columns where `col`) of a matrix.
Operand rows_of(const Matrix& m) { return Operand{{m.p, nullptr}, m.ld, m.plane, m.rows, m.cols}; }
Operand columns_of(const Matrix& m) { return Operand{{m.p, nullptr}, m.ld, m.plane, m.cols, m.rows}; }

// G, U (kept where `saved`) and H (where `h`).
template <class T, int HP>
void run_gate(const fd_gated_block& b, const Work& w, const Matrix& x, const Matrix& wg,
              const Matrix& wu, char* saved, bool h, hipStream_t st) {
  GemmArgs p{};
  p.a = rows_of(x);
  p.b = rows_of(wg);
  p.up = wu.p;
  p.M = b.N;
  p.N = b.F;
  p.segs = 1;
  p.ktiles = ceil_div(x.cols, k_tile<T>);
  p.bg = b.bg;
  p.bu = b.bu;
  p.saved = saved;
  p.Fp = f_padded(b.F);
  p.H = h ? w.h : nullptr;
  p.hplane = b.N * p.Fp;
  const auto run = activation_of(b) == FD_ACT_SILU ? launch_inner<false, GATE, T, FD_ACT_SILU, HP>
                                        : launch_inner<false, GATE, T, FD_ACT_GELU, HP>;
  run(w.plan.gate_config, w.plan.gate, w.part, p, st);
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
  FD_REQUIRE(activation_of(b) == FD_ACT_SILU || activation_of(b) == FD_ACT_GELU,
             FD_ERR_INVALID_ARG, "unknown activation");
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
  FD_REQUIRE(bytes >= saved_bytes(b), FD_ERR_WORKSPACE,
             "saved is too small");
  FD_REQUIRE((reinterpret_cast<uintptr_t>(saved) & 255) == 0, FD_ERR_WORKSPACE,
             "saved must be 256-byte aligned");
}

Work carve_checked(const fd_gated_block& b, int backward, void* ws, size_t ws_bytes) {
  check_workspace(ws, ws_bytes, 1);
  Arena a;
  a.base = static_cast<char*>(ws);
  a.cap = ws_bytes;
  return carve_work(a, b, backward);  // throws where it does not fit
}

template <class T>
int grad_wave_rows(int config) {
  if (config == BIG) return Config<BIG, GRAD, T>::wm;
  return config == MID ? Config<MID, GRAD, T>::wm : Config<SMALL, GRAD, T>::wm;
}

// Both inner weights, laid out alike.
void bring_weights(Work& w, const fd_gated_block& b, Matrix& wg, Matrix& wu) {
  const int t = b.type;
  if (direct(b.Wg, b.ldwi, b.D, t) && direct(b.Wu, b.ldwi, b.D, t)) {
    wg = bring(w, b.Wg, b.ldwi, b.F, b.D, t, w.wg);
    wu = bring(w, b.Wu, b.ldwi, b.F, b.D, t, w.wu);
  } else {
    wg = pack(w, b.Wg, b.ldwi, b.F, b.D, w.wg);
    wu = pack(w, b.Wu, b.ldwi, b.F, b.D, w.wu);
  }
}

template <class T, int HP>
void forward(const fd_gated_block& b, Work& w, const void* R, int64_t ldr, void* Y, int64_t ldy,
             char* saved, hipStream_t st) {
  const int t = b.type;
  const Way way = forward_way(b.N, b.D, b.O, sizeof(T) == 4, saved != nullptr);
  if (way == FEW_ROWS) {
    const int64_t Fp = f_padded(b.F), plane = b.N * Fp;
    SkinnyArgs p{b.X,  b.Wg,    b.Wu, b.ldx, b.ldwi, b.N, b.F, b.D,
                 b.bg, b.bu, nullptr,     0,    w.h,  Fp,   0, plane};
    constexpr int SP = sizeof(T) == 4 ? 1 : HP;
    if (activation_of(b) == FD_ACT_SILU) launch_skinny<T, SP, true, FD_ACT_SILU>(p, st);
    else launch_skinny<T, SP, true, FD_ACT_GELU>(p, st);
    p = SkinnyArgs{w.h,  b.Wd,    nullptr, Fp,  b.ldwd, b.N, b.O,   b.F,
                   b.bd, nullptr, R,       ldr, Y,      ldy, plane, 0};
    launch_skinny<T, SP, false, 0>(p, st);
    return;
  }
  if (way == NARROW_WAY) {
    NarrowArgs p{b,      R,    ldr, Y, ldy, saved, f_padded(b.F), narrow_parts(b.N, b.F),
                 w.part, round_up(b.O, 4)};
    p.b.act = activation_of(b);
    run_narrow(p, HP, st);
    if (p.parts == 1) return;
    AfterJobs after;
    after.splits = 1;
    after.s[0] = SplitJob{p.part, p.parts, b.N, b.O, p.ldp, {Y, nullptr}, ldy, b.N, b.N, b.bd, R, ldr, 0};
    after.groups = ceil_div(b.N * ceil_div(b.O, 4), GROUP);
    run_after<T>(after, st);
    return;
  }
  const Matrix x = bring(w, b.X, b.ldx, b.N, b.D, t, w.x);
  Matrix wg, wu;
  bring_weights(w, b, wg, wu);
  const Matrix wd = bring(w, b.Wd, b.ldwd, b.O, b.F, t, w.wd);
  run_before<T>(w.jobs, st);
  run_gate<T, HP>(b, w, x, wg, wu, saved, true, st);
  const int64_t Fp = f_padded(b.F);
  GemmArgs p{};
  p.a = rows_of(Matrix{w.h, Fp, b.N, Fp, b.N * Fp});
  p.b = rows_of(wd);
  p.M = b.N;
  p.N = b.O;
  p.segs = 1;
  p.ktiles = Fp / k_tile<T>;
  p.out[0] = Y;
  p.ldo = ldy;
  p.half = p.rows = b.N;
  p.bias = b.bd;
  p.R = R;
  p.ldr = ldr;
  AfterJobs after;
  float* room = w.part;
  set_parts(p, w.plan.out[0], room, after);
  launch<false, false, STORE, T, 0, HP>(w.plan.config, p, st);
  run_after<T>(after, st);
}

template <class T>
void clear(void* p, int64_t rows, int64_t cols, int64_t ld, hipStream_t st) {
  if (p == nullptr) return;
  const int64_t groups = std::min<int64_t>(ceil_div(rows * cols, GROUP), 1 << 16);
  clear_kernel<T><<<dim3(unsigned(groups)), dim3(GROUP), 0, st>>>(static_cast<T*>(p), rows, cols, ld);
  FD_LAUNCH_CHECK();
}

template <class T, int HP>
void backward(const fd_gated_block& b, Work& w, const void* dY, int64_t lddy, char* saved,
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
  const bool gate = inner && saved == nullptr;
  const bool inner_weights = g.dWg != nullptr || g.dWu != nullptr;
  Matrix x, wg, wu, wd, dy;
  if (gate || inner_weights) x = bring(w, b.X, b.ldx, b.N, b.D, t, w.x);
  if (gate || g.dX != nullptr) bring_weights(w, b, wg, wu);
  if (inner) {
    wd = bring(w, b.Wd, b.ldwd, b.O, b.F, t, w.wd);
    dy = bring(w, dY, lddy, b.N, b.O, t, w.dy);
  }
  AfterJobs after;
  const int64_t parts = std::min<int64_t>(SUM_PARTS, ceil_div(b.N, 16));
  if (g.dbd != nullptr) {
    w.jobs.sum = dY;
    w.jobs.sum_ld = lddy;
    w.jobs.sum_rows = b.N;
    w.jobs.sum_cols = b.O;
    w.jobs.sum_parts = parts;
    w.jobs.sum_out = w.dysum;
  }
  run_before<T>(w.jobs, st);
  GemmGroup group{};
  if (inner) {
    if (gate) {
      run_gate<T, HP>(b, w, x, wg, wu, w.saved, false, st);
      saved = w.saved;
    }
    GemmArgs p{};  // dH, and from it dG, dU, H
    p.a = rows_of(dy);
    p.b = columns_of(wd);
    p.M = b.N;
    p.N = b.F;
    p.segs = 1;
    p.ktiles = ceil_div(b.O, k_tile<T>);
    p.saved = saved;
    p.Fp = Fp;
    p.H = w.h;
    p.hplane = b.N * Fp;
    p.dGU = w.dgu;
    p.gplane = b.N * 2 * Fp;
    p.colsum = g.dbg != nullptr || g.dbu != nullptr ? w.colsum : nullptr;
    const auto run = activation_of(b) == FD_ACT_SILU ? launch_inner<true, GRAD, T, FD_ACT_SILU, HP>
                                          : launch_inner<true, GRAD, T, FD_ACT_GELU, HP>;
    run(w.plan.grad_config, w.plan.grad, w.part, p, st);
    const int64_t sum_rows = w.plan.grad.splits > 1
                                 ? ceil_div(b.N, 32)
                                 : p.tiles_m * grad_wave_rows<T>(w.plan.grad_config);

    const Matrix h{w.h, Fp, b.N, Fp, b.N * Fp}, dgu{w.dgu, 2 * Fp, b.N, 2 * Fp, b.N * 2 * Fp};
    Shape shapes[GROUP_GEMMS];
    if (g.dX != nullptr) {  // [dG dU] [Wg; Wu]
      GemmArgs& q = group.g[group.count];
      q.a = rows_of(dgu);
      q.a.k = Fp;
      q.a.p[1] = w.dgu + Fp;
      q.b = columns_of(wg);
      q.b.p[1] = wu.p;
      q.segs = 2;
      q.ktiles = Fp / k_tile<T>;
      q.out[0] = g.dX;
      q.ldo = g.lddx;
      q.half = q.rows = b.N;
      shapes[group.count++] = w.plan.out[0];
    }
    if (inner_weights) {  // [dG dU]^T X
      GemmArgs& q = group.g[group.count];
      q.a = columns_of(dgu);
      q.b = columns_of(x);
      q.segs = 1;
      q.ktiles = ceil_div(b.N, k_tile<T>);
      q.out[0] = g.dWg;
      q.out[1] = g.dWu;
      q.ldo = g.lddwi;
      q.half = Fp;
      q.rows = b.F;
      group.acol[group.count] = true;
      shapes[group.count++] = w.plan.out[1];
    }
    if (g.dWd != nullptr) {  // dY^T H
      GemmArgs& q = group.g[group.count];
      q.a = columns_of(dy);
      q.b = columns_of(h);
      q.segs = 1;
      q.ktiles = ceil_div(b.N, k_tile<T>);
      q.out[0] = g.dWd;
      q.ldo = g.lddwd;
      q.half = q.rows = b.O;
      group.acol[group.count] = group.inner[group.count] = true;
      shapes[group.count++] = w.plan.out[2];
    }
    if (group.count > 0) {
      float* room = w.part;
      for (int i = 0; i < group.count; ++i) {
        group.g[i].M = shapes[i].M;
        group.g[i].N = shapes[i].N;
        set_parts(group.g[i], shapes[i], room, after);
      }
      auto run = launch_group<SMALL, T, HP>;
      if constexpr (HP == planes_of<T>) {
        if (w.plan.config == BIG) run = launch_group<BIG, T, HP>;
        if (w.plan.config == MID) run = launch_group<MID, T, HP>;
      }
      run(group, st);
    }
    if (g.dbg != nullptr || g.dbu != nullptr)
      add_columns(after, w.colsum, sum_rows, 2 * Fp, Fp, b.F, g.dbg, g.dbu);
  }
  if (g.dbd != nullptr) add_columns(after, w.dysum, parts, b.O, b.O, b.O, g.dbd, nullptr);
  run_after<T>(after, st);
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
    out = saved_bytes(*b);
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
      forward<float, 3>(*b, w, R, ldr, Y, ldy, static_cast<char*>(saved), st);
    else if (fine(*b))
      forward<bf16, 2>(*b, w, R, ldr, Y, ldy, static_cast<char*>(saved), st);
    else
      forward<bf16, 1>(*b, w, R, ldr, Y, ldy, static_cast<char*>(saved), st);
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
    char* kept = static_cast<char*>(const_cast<void*>(saved));
    if (b->type == FD_F32)
      backward<float, 3>(*b, w, dY, lddy, kept, g, st);
    else if (fine(*b))
      backward<bf16, 2>(*b, w, dY, lddy, kept, g, st);
    else
      backward<bf16, 1>(*b, w, dY, lddy, kept, g, st);
  });
}

}  // extern "C"
