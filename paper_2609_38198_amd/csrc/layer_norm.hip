// Layer norm over the features of each row, forward and backward.
#include <algorithm>
#include <cmath>

#include "fd_guard.hpp"
#include "fd_solver.hpp"
#include "net_common.hpp"

namespace fd {
namespace net {
namespace {

constexpr int GROUP = 256;         // threads of a workgroup, except the widest rows'
constexpr int64_t PARTS = 768;     // workgroups of a backward pass, each with its own partial sums

// A row is held in registers by L lanes (16 or 64: part of a wave; 256 or
// 1024: a workgroup), C chunks of 16 bytes each: lane l has chunks l, l + L, ...
// so that each access of the group is contiguous.
template <int L>
constexpr int threads_of = L > GROUP ? L : GROUP;

// Sums of two values over the L lanes of a row.  red: 2 x 16 floats.
template <int L>
__device__ __forceinline__ void row_sum2(float& a, float& b, float* red) {
  a = lane_sum<(L < WAVE ? L : WAVE)>(a);
  b = lane_sum<(L < WAVE ? L : WAVE)>(b);
  if (L > WAVE) {
    constexpr int W = L > WAVE ? L / WAVE : 1;
    const int wave = threadIdx.x / WAVE;
    __syncthreads();
    if (threadIdx.x % WAVE == 0) {
      red[wave] = a;
      red[16 + wave] = b;
    }
    __syncthreads();
    a = b = 0.f;
    for (int i = 0; i < W; ++i) {
      a += red[i];
      b += red[16 + i];
    }
  }
}

template <int C, int V, int L, class T>
__device__ __forceinline__ void load_row(const T* p, int lane, int D, float (&x)[C * V]) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * L + lane) * V;
    load_wide<V>(p + at, D - at, x + c * V);
  }
}

template <int C, int V, int L, class T>
__device__ __forceinline__ void store_row(T* p, int lane, int D, const float (&x)[C * V]) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * L + lane) * V;
    store_wide<V>(p + at, D - at, x + c * V);
  }
}

// Features of a wt array, or `fill` where there is none.
template <int C, int V, int L, class W>
__device__ __forceinline__ void load_weight(const W* p, int lane, int D, float fill,
                                            float (&x)[C * V]) {
  if (p != nullptr) {
    load_row<C, V, L>(p, lane, D, x);
  } else {
#pragma unroll
    for (int i = 0; i < C * V; ++i) x[i] = fill;
  }
}

// One read and one write of each element; the variance is summed from the
// centred values, which are in registers, so rows far from zero keep their
// digits.  gamma and beta stay in registers over the rows of a workgroup.
template <class T, class W, int L, int C>
__global__ __launch_bounds__(threads_of<L>) void norm_kernel(
    const T* X, int64_t N, int D, int64_t ldx, const W* gamma, const W* beta, float eps, T* Y,
    int64_t ldy, float2* stats) {
  constexpr int V = VEC<T>;
  __shared__ float red[32];
  const int lane = threadIdx.x % L, sub = threadIdx.x / L;
  constexpr int ROWS = threads_of<L> / L;
  float ga[C * V], be[C * V], x[C * V];
  load_weight<C, V, L>(gamma, lane, D, 1.f, ga);
  load_weight<C, V, L>(beta, lane, D, 0.f, be);
  const float inv = 1.f / float(D);
  for (int64_t r0 = int64_t(blockIdx.x) * ROWS; r0 < N; r0 += int64_t(gridDim.x) * ROWS) {
    const int64_t row = r0 + sub;
    const bool live = row < N;
    load_row<C, V, L>(X + (live ? row : N - 1) * ldx, lane, D, x);
    float s = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < C * V; ++i) s += x[i];
    row_sum2<L>(s, none, red);
    const float mean = s * inv;
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = x[c * V + i] - mean;
        x[c * V + i] = d;
        if ((c * L + lane) * V + i < D) q += d * d;
      }
    none = 0.f;
    row_sum2<L>(q, none, red);
    const float rstd = 1.f / sqrtf(q * inv + eps);
#pragma unroll
    for (int i = 0; i < C * V; ++i) x[i] = x[i] * rstd * ga[i] + be[i];
    if (live) {
      store_row<C, V, L>(Y + row * ldy, lane, D, x);
      if (stats != nullptr && lane == 0) stats[row] = make_float2(mean, rstd);
    }
  }
}

// dx row by row as above, and dgamma, dbeta summed in registers over the
// workgroup's rows; the groups of a workgroup are then added in LDS and each
// workgroup writes 2 D partial sums, so that the total has one fixed order.
template <class T, class W, int L, int C>
__global__ __launch_bounds__(threads_of<L>) void norm_backward_kernel(
    const T* dY, int64_t lddy, const T* X, int64_t N, int D, int64_t ldx, const W* gamma,
    const float2* stats, const T* add, int64_t ldadd, T* dX, int64_t lddx, float* part) {
  constexpr int V = VEC<T>;
  constexpr int ROWS = threads_of<L> / L;
  __shared__ float red[32];
  const int lane = threadIdx.x % L, sub = threadIdx.x / L;
  float ga[C * V], dga[C * V], dbe[C * V];
  load_weight<C, V, L>(gamma, lane, D, 1.f, ga);
#pragma unroll
  for (int i = 0; i < C * V; ++i) dga[i] = dbe[i] = 0.f;
  const float inv = 1.f / float(D);
  for (int64_t r0 = int64_t(blockIdx.x) * ROWS; r0 < N; r0 += int64_t(gridDim.x) * ROWS) {
    const int64_t row = r0 + sub;
    const bool live = row < N;
    const int64_t at = live ? row : N - 1;
    float x[C * V], g[C * V];
    load_row<C, V, L>(X + at * ldx, lane, D, x);
    load_row<C, V, L>(dY + at * lddy, lane, D, g);
    const float2 st = stats[at];
    float s = 0.f, sh = 0.f;
#pragma unroll
    for (int i = 0; i < C * V; ++i) {
      const float h = (x[i] - st.x) * st.y;  // past the row's end g is zero
      if (live) {
        dga[i] += g[i] * h;
        dbe[i] += g[i];
      }
      g[i] *= ga[i];
      s += g[i];
      sh += g[i] * h;
      x[i] = h;
    }
    row_sum2<L>(s, sh, red);
    s *= inv;
    sh *= inv;
#pragma unroll
    for (int i = 0; i < C * V; ++i) g[i] = st.y * (g[i] - s - x[i] * sh);
    if (live) {
      if (add != nullptr) {
        load_row<C, V, L>(add + row * ldadd, lane, D, x);
#pragma unroll
        for (int i = 0; i < C * V; ++i) g[i] += x[i];
      }
      store_row<C, V, L>(dX + row * lddx, lane, D, g);
    }
  }
  if (part == nullptr) return;
  // the workgroup's rows in a fixed order: group 0, then 1, ...
  __shared__ float sums[ROWS > 1 ? 2 * L * C * V : 1];
  for (int r = 0; r < ROWS; ++r) {
    if (ROWS > 1) __syncthreads();
    if (sub == r) {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int f = (c * L + lane) * V + i;
          float a = dga[c * V + i], b = dbe[c * V + i];
          if (ROWS > 1) {
            if (r > 0) {
              a += sums[f];
              b += sums[L * C * V + f];
            }
            sums[f] = a;
            sums[L * C * V + f] = b;
          }
          if (r == ROWS - 1 && f < D) {
            part[int64_t(blockIdx.x) * 2 * D + f] = a;
            part[int64_t(blockIdx.x) * 2 * D + D + f] = b;
          }
        }
    }
  }
}

// Column sums of `rows` x 2 D partial sums: 16 columns a workgroup, 16 rows at
// a time, the sixteen running sums added in order.
template <class W>
__global__ __launch_bounds__(GROUP) void norm_reduce_kernel(const float* part, int64_t rows,
                                                            int64_t D, W* dgamma, W* dbeta) {
  __shared__ float sums[16][17];
  const int c = threadIdx.x % 16, r = threadIdx.x / 16;
  const int64_t col = int64_t(blockIdx.x) * 16 + c;
  float s = 0.f;
  if (col < 2 * D)
    for (int64_t i = r; i < rows; i += 16) s += part[i * 2 * D + col];
  sums[r][c] = s;
  __syncthreads();
  if (r != 0 || col >= 2 * D) return;
  for (int i = 1; i < 16; ++i) s += sums[i][c];
  W* out = col < D ? dgamma : dbeta;
  if (out != nullptr) out[col < D ? col : col - D] = narrow<W>(s);
}

// Rows too wide for registers (above 16,384 features): one workgroup per row reads it once for each sum.
__device__ __forceinline__ float wide_sum(float s, float* red) {
  float none = 0.f;
  row_sum2<GROUP>(s, none, red);
  return s;
}

template <class T, class W>
__global__ __launch_bounds__(GROUP) void norm_wide_kernel(const T* X, int64_t N, int64_t D,
                                                          int64_t ldx, const W* gamma,
                                                          const W* beta, float eps, T* Y,
                                                          int64_t ldy, float2* stats) {
  __shared__ float red[32];
  const float inv = 1.f / float(D);
  for (int64_t row = blockIdx.x; row < N; row += gridDim.x) {
    const T* x = X + row * ldx;
    float s = 0.f;
    for (int64_t i = threadIdx.x; i < D; i += GROUP) s += widen(x[i]);
    const float mean = wide_sum(s, red) * inv;
    s = 0.f;
    for (int64_t i = threadIdx.x; i < D; i += GROUP) {
      const float d = widen(x[i]) - mean;
      s += d * d;
    }
    const float rstd = 1.f / sqrtf(wide_sum(s, red) * inv + eps);
    for (int64_t i = threadIdx.x; i < D; i += GROUP) {
      const float ga = gamma != nullptr ? widen(gamma[i]) : 1.f;
      const float be = beta != nullptr ? widen(beta[i]) : 0.f;
      Y[row * ldy + i] = narrow<T>((widen(x[i]) - mean) * rstd * ga + be);
    }
    if (stats != nullptr && threadIdx.x == 0) stats[row] = make_float2(mean, rstd);
  }
}

template <class T, class W>
__global__ __launch_bounds__(GROUP) void norm_wide_backward_kernel(
    const T* dY, int64_t lddy, const T* X, int64_t N, int64_t D, int64_t ldx, const W* gamma,
    const float2* stats, const T* add, int64_t ldadd, T* dX, int64_t lddx) {
  __shared__ float red[32];
  const float inv = 1.f / float(D);
  for (int64_t row = blockIdx.x; row < N; row += gridDim.x) {
    const T* x = X + row * ldx;
    const T* dy = dY + row * lddy;
    const float2 st = stats[row];
    float s = 0.f, sh = 0.f;
    for (int64_t i = threadIdx.x; i < D; i += GROUP) {
      const float g = widen(dy[i]) * (gamma != nullptr ? widen(gamma[i]) : 1.f);
      s += g;
      sh += g * ((widen(x[i]) - st.x) * st.y);
    }
    row_sum2<GROUP>(s, sh, red);
    s *= inv;
    sh *= inv;
    for (int64_t i = threadIdx.x; i < D; i += GROUP) {
      const float g = widen(dy[i]) * (gamma != nullptr ? widen(gamma[i]) : 1.f);
      float d = st.y * (g - s - (widen(x[i]) - st.x) * st.y * sh);
      if (add != nullptr) d += widen(add[row * ldadd + i]);
      dX[row * lddx + i] = narrow<T>(d);
    }
  }
}

// dgamma, dbeta of wide rows: a thread per feature, before dX (which may be dY).
template <class T, class W>
__global__ __launch_bounds__(GROUP) void norm_wide_weight_kernel(
    const T* dY, int64_t lddy, const T* X, int64_t N, int64_t D, int64_t ldx, const float2* stats,
    W* dgamma, W* dbeta) {
  const int64_t f = int64_t(blockIdx.x) * GROUP + threadIdx.x;
  if (f >= D) return;
  float a = 0.f, b = 0.f;
  for (int64_t row = 0; row < N; ++row) {
    const float g = widen(dY[row * lddy + f]);
    a += g * ((widen(X[row * ldx + f]) - stats[row].x) * stats[row].y);
    b += g;
  }
  if (dgamma != nullptr) dgamma[f] = narrow<W>(a);
  if (dbeta != nullptr) dbeta[f] = narrow<W>(b);
}

struct Forward {
  const void* X;
  int64_t N, D, ldx;
  const void *gamma, *beta;
  float eps;
  void* Y;
  int64_t ldy;
  float2* stats;
  hipStream_t stream;

  template <class T, class W, int L, int C>
  void run() const {
    constexpr int64_t ROWS = threads_of<L> / L;
    const int64_t grid = std::min<int64_t>(ceil_div(N, ROWS), 8192);
    norm_kernel<T, W, L, C><<<dim3(unsigned(grid)), dim3(threads_of<L>), 0, stream>>>(
        static_cast<const T*>(X), N, int(D), ldx, static_cast<const W*>(gamma),
        static_cast<const W*>(beta), eps, static_cast<T*>(Y), ldy, stats);
  }
  template <class T, class W>
  void wide() const {
    norm_wide_kernel<T, W><<<dim3(unsigned(std::min<int64_t>(N, 8192))), dim3(GROUP), 0, stream>>>(
        static_cast<const T*>(X), N, D, ldx, static_cast<const W*>(gamma),
        static_cast<const W*>(beta), eps, static_cast<T*>(Y), ldy, stats);
  }
};

int64_t norm_parts(int64_t N) { return std::min<int64_t>(N, PARTS); }

struct Backward {
  const void* dY;
  int64_t lddy;
  const void* X;
  int64_t N, D, ldx;
  const void* gamma;
  const float2* stats;
  const void* add;
  int64_t ldadd;
  void* dX;
  int64_t lddx;
  void *dgamma, *dbeta;
  float* part;
  hipStream_t stream;

  template <class T, class W, int L, int C>
  void run() const {
    constexpr int64_t ROWS = threads_of<L> / L;
    const int64_t grid = std::min<int64_t>(ceil_div(N, ROWS), norm_parts(N));
    const bool weights = dgamma != nullptr || dbeta != nullptr;
    norm_backward_kernel<T, W, L, C><<<dim3(unsigned(grid)), dim3(threads_of<L>), 0, stream>>>(
        static_cast<const T*>(dY), lddy, static_cast<const T*>(X), N, int(D), ldx,
        static_cast<const W*>(gamma), stats, static_cast<const T*>(add), ldadd,
        static_cast<T*>(dX), lddx, weights ? part : nullptr);
    FD_LAUNCH_CHECK();
    if (weights)
      norm_reduce_kernel<W><<<dim3(unsigned(ceil_div(2 * D, 16))), dim3(GROUP), 0, stream>>>(
          part, grid, D, static_cast<W*>(dgamma), static_cast<W*>(dbeta));
  }
  template <class T, class W>
  void wide() const {
    if (dgamma != nullptr || dbeta != nullptr) {
      norm_wide_weight_kernel<T, W>
          <<<dim3(unsigned(ceil_div(D, GROUP))), dim3(GROUP), 0, stream>>>(
              static_cast<const T*>(dY), lddy, static_cast<const T*>(X), N, D, ldx, stats,
              static_cast<W*>(dgamma), static_cast<W*>(dbeta));
      FD_LAUNCH_CHECK();
    }
    norm_wide_backward_kernel<T, W>
        <<<dim3(unsigned(std::min<int64_t>(N, 8192))), dim3(GROUP), 0, stream>>>(
            static_cast<const T*>(dY), lddy, static_cast<const T*>(X), N, D, ldx,
            static_cast<const W*>(gamma), stats, static_cast<const T*>(add), ldadd,
            static_cast<T*>(dX), lddx);
  }
};

// The narrowest group of lanes that holds a row: in units of V elements, 16
// lanes x 1 chunk up to 1,024 lanes x 16 elements (more would spill).
template <class T, class W, class Call>
void by_width(const Call& call) {
  const int64_t chunks = ceil_div(call.D, VEC<T>);
  if (chunks <= 16) call.template run<T, W, 16, 1>();
  else if (chunks <= 64) call.template run<T, W, 64, 1>();
  else if (chunks <= 128) call.template run<T, W, 64, 2>();
  else if (chunks <= 256) call.template run<T, W, 64, 4>();
  else if (chunks <= 512) call.template run<T, W, 256, 2>();
  else if (chunks <= 1024) call.template run<T, W, 256, 4>();
  else if (chunks <= 2048) call.template run<T, W, 1024, 2>();
  else if (chunks <= 16384 / VEC<T>) call.template run<T, W, 1024, 16 / VEC<T>>();
  else call.template wide<T, W>();
  FD_LAUNCH_CHECK();
}

template <class Call>
void by_type(int xt, int wt, const Call& call) {
  if (xt == FD_F32 && wt == FD_F32) by_width<float, float>(call);
  else if (xt == FD_F32) by_width<float, bf16>(call);
  else if (wt == FD_F32) by_width<bf16, float>(call);
  else by_width<bf16, bf16>(call);
}

void check_norm(const void* X, int xt, int64_t N, int64_t D, int64_t ldx, const void* gamma,
                const void* beta, int wt) {
  check_dtype(xt, "dtype");
  check_dtype(wt, "weight dtype");
  FD_REQUIRE(N >= 0 && N <= MAX_ROWS, FD_ERR_INVALID_ARG, "N out of range [0, 2^30]");
  FD_REQUIRE(D >= 1 && D <= MAX_WIDTH, FD_ERR_INVALID_ARG, "D out of range [1, 2^20]");
  FD_REQUIRE(ldx >= D, FD_ERR_INVALID_ARG, "ldx must be >= D");
  FD_REQUIRE(N == 0 || X != nullptr, FD_ERR_INVALID_ARG, "X is NULL");
  check_element_aligned(X, xt, "X");
  check_element_aligned(gamma, wt, "gamma");
  check_element_aligned(beta, wt, "beta");
}

}  // namespace
}  // namespace net
}  // namespace fd

using namespace fd;
using namespace fd::net;

extern "C" {

fd_status fd_layer_norm(const void* X, fd_dtype xt, int64_t N, int64_t D, int64_t ldx,
                        const void* gamma, const void* beta, fd_dtype wt, float eps, void* Y,
                        int64_t ldy, float* stats, void* stream) {
  return guarded([&] {
    check_norm(X, xt, N, D, ldx, gamma, beta, wt);
    FD_REQUIRE(N == 0 || Y != nullptr, FD_ERR_INVALID_ARG, "Y is NULL");
    FD_REQUIRE(ldy >= D, FD_ERR_INVALID_ARG, "ldy must be >= D");
    FD_REQUIRE(Y != X || N == 0 || ldy == ldx, FD_ERR_INVALID_ARG, "Y = X needs ldy = ldx");
    FD_REQUIRE(std::isfinite(eps) && eps >= 0.f, FD_ERR_INVALID_ARG, "eps must be finite and >= 0");
    FD_REQUIRE((reinterpret_cast<uintptr_t>(stats) & 7) == 0, FD_ERR_INVALID_ARG,
               "stats must be 8-byte aligned");
    check_element_aligned(Y, xt, "Y");
    if (N == 0) return;
    by_type(xt, wt, Forward{X, N, D, ldx, gamma, beta, eps, Y, ldy,
                            reinterpret_cast<float2*>(stats), static_cast<hipStream_t>(stream)});
  });
}

size_t fd_layer_norm_workspace_size(int64_t N, int64_t D) {
  if (N < 0 || N > MAX_ROWS || D < 1 || D > MAX_WIDTH) return 0;
  return size_t(std::max<int64_t>(norm_parts(N), 1) * 2 * D) * sizeof(float);
}

fd_status fd_layer_norm_backward(const void* dY, int64_t lddy, const void* X, fd_dtype xt,
                                 int64_t N, int64_t D, int64_t ldx, const void* gamma, fd_dtype wt,
                                 const float* stats, const void* add, int64_t ldadd, void* dX,
                                 int64_t lddx, void* dgamma, void* dbeta, void* ws,
                                 size_t ws_bytes, void* stream) {
  return guarded([&] {
    check_norm(X, xt, N, D, ldx, gamma, nullptr, wt);
    FD_REQUIRE(N == 0 || (dY != nullptr && dX != nullptr && stats != nullptr), FD_ERR_INVALID_ARG,
               "dY, dX and stats must not be NULL");
    FD_REQUIRE(lddy >= D && lddx >= D && (add == nullptr || ldadd >= D), FD_ERR_INVALID_ARG,
               "leading dimensions must be >= D");
    FD_REQUIRE(N == 0 || ((dX != dY || lddx == lddy) && (dX != add || lddx == ldadd)),
               FD_ERR_INVALID_ARG, "dX in place needs equal leading dimensions");
    FD_REQUIRE((reinterpret_cast<uintptr_t>(stats) & 7) == 0, FD_ERR_INVALID_ARG,
               "stats must be 8-byte aligned");
    check_element_aligned(dY, xt, "dY");
    check_element_aligned(dX, xt, "dX");
    check_element_aligned(add, xt, "add");
    check_element_aligned(dgamma, wt, "dgamma");
    check_element_aligned(dbeta, wt, "dbeta");
    check_workspace(ws, ws_bytes, fd_layer_norm_workspace_size(N, D));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (N == 0) {  // sums over no rows
      const unsigned grid = unsigned(ceil_div(2 * D, 16));
      if (wt == FD_F32)
        norm_reduce_kernel<float><<<dim3(grid), dim3(GROUP), 0, st>>>(
            nullptr, 0, D, static_cast<float*>(dgamma), static_cast<float*>(dbeta));
      else
        norm_reduce_kernel<bf16><<<dim3(grid), dim3(GROUP), 0, st>>>(
            nullptr, 0, D, static_cast<bf16*>(dgamma), static_cast<bf16*>(dbeta));
      FD_LAUNCH_CHECK();
      return;
    }
    by_type(xt, wt, Backward{dY, lddy, X, N, D, ldx, gamma, reinterpret_cast<const float2*>(stats),
                             add, ldadd, dX, lddx, dgamma, dbeta, static_cast<float*>(ws), st});
  });
}

}  // extern "C"
