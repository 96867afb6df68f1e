// Layer norm over the features of each row, forward and backward.
#include <algorithm>
#include <cmath>

#include "fd_guard.hpp"
#include "fd_solver.hpp"
#include "net_common.hpp"

namespace fd {
namespace net {
namespace {

constexpr int GROUP = 256;         // threads of a forward workgroup, except the widest rows'
constexpr int WIDE_GROUP = 1024;   // and of a backward one: one to a CU
constexpr int64_t PARTS = 256;     // backward workgroups at most, each with its own partial sums

// A row is held in registers by L lanes (16 or 64: part of a wave; more: several
// waves), C chunks of 16 bytes each: lane l has chunks l, l + L, ... so that
// each access of the group is contiguous.  R rows are on their way at once.
template <class T>
struct Chunk {
  T v[VEC<T>];
};

// Leaves a chunk as it is, but the compiler with only its 16 bytes: what was widened from
// it is widened again rather than kept in four times the registers.
template <class T>
__device__ __forceinline__ void keep_narrow(Chunk<T>& c) {
  typedef int intx4 __attribute__((ext_vector_type(4)));
  intx4 w = __builtin_bit_cast(intx4, c);
  asm volatile("" : "+v"(w));
  c = __builtin_bit_cast(Chunk<T>, w);
}

// The group of L lanes that a thread is in: uniform where it is whole waves.
template <int L>
__device__ __forceinline__ int row_group() {
  const int g = threadIdx.x / L;
  return L < WAVE ? g : __builtin_amdgcn_readfirstlane(g);
}

// Chunk c of a lane.  EVEN: rows are whole chunks, and one is there or not.
// Else the chunk at a row's end (and those past it) lies where it is still
// whole, over the end of the one before it: `skip` of its values are that
// one's and do not count, though both lanes make and store the same results.
template <int L, int V, bool EVEN>
struct Place {
  int at, skip;
  bool there;
  __device__ __forceinline__ Place(int c, int lane, int D) {
    const int want = (c * L + lane) * V;
    there = want < D;
    at = EVEN ? want : min(want, D - V);
    skip = want - at;
  }
  __device__ __forceinline__ bool counts(int i) const { return EVEN ? there : i >= skip; }
};
template <int L, bool EVEN, class T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, const Place<L, VEC<T>, EVEN>& w) {
  Chunk<T> c = {};
  if (!EVEN || w.there) __builtin_memcpy(&c, p + w.at, 16);
  return c;
}
template <int L, bool EVEN, class T>
__device__ __forceinline__ void store_chunk(T* p, const Place<L, VEC<T>, EVEN>& w,
                                            const Chunk<T>& c) {
  if (w.there) __builtin_memcpy(p + w.at, &c, 16);
}
// V features of a weight of type W, or `fill` where there is none.
template <int L, int V, bool EVEN, class W>
__device__ __forceinline__ void load_weight(const W* p, const Place<L, V, EVEN>& w, float fill,
                                            float* out) {
  if (p != nullptr) {
    load_wide<V>(p + w.at, EVEN && !w.there ? 0 : V, out);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = fill;
  }
}

// Sums over the L lanes of a row, in every lane.  Rows of several waves meet in
// LDS, in one of two places in turn: a place is written again only after the
// barrier of the call in between, which its readers have passed.
template <int L, int K, int WAVES>
__device__ __forceinline__ void row_sums(float (&x)[K], float (*red)[K][WAVES], int& turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) x[k] = lane_sum<(L < WAVE ? L : WAVE)>(x[k]);
  if (L <= WAVE) return;
  constexpr int N = L > WAVE ? L / WAVE : 1;
  const int wave = threadIdx.x / WAVE;
  if (threadIdx.x % WAVE == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) red[turn][k][wave] = x[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k)
    x[k] = lane_sum<N>(red[turn][k][wave / N * N + threadIdx.x % N]);
  turn ^= 1;
}

// One read and one write of each element; the variance is summed from the
// centred values, which are in registers, so rows far from zero keep their
// digits.  65,536 x 2,048 bfloat16: 91 us, 5.9 TB/s on
// one set of inputs; 30,011 x 301 float32: 16 us.
template <class T, class W, int L, int C, int R, bool EVEN>
__global__ __launch_bounds__(L > GROUP ? L : GROUP) void norm_kernel(
    const T* X, int64_t N, int D, int64_t ldx, const W* gamma, const W* beta, float eps, T* Y,
    int64_t ldy, float2* stats) {
  constexpr int THREADS = L > GROUP ? L : GROUP, V = VEC<T>, ROWS = THREADS / L * R;
  __shared__ float red[2][R][THREADS / WAVE];
  const int lane = threadIdx.x % L, sub = row_group<L>();
  const float inv = 1.f / float(D);
  int turn = 0;
  for (int64_t r0 = int64_t(blockIdx.x) * ROWS; r0 < N; r0 += int64_t(gridDim.x) * ROWS) {
    Chunk<T> raw[R][C];
    float mean[R], q[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = min(r0 + sub * R + r, N - 1);
#pragma unroll
      for (int c = 0; c < C; ++c)
        raw[r][c] = load_chunk<L, EVEN>(X + row * ldx, Place<L, V, EVEN>(c, lane, D));
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean[r] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Place<L, V, EVEN> w(c, lane, D);
#pragma unroll
        for (int i = 0; i < V; ++i) mean[r] += EVEN || w.counts(i) ? widen(raw[r][c].v[i]) : 0.f;
      }
    }
    row_sums<L>(mean, red, turn);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean[r] *= inv;
      q[r] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Place<L, V, EVEN> w(c, lane, D);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = widen(raw[r][c].v[i]) - mean[r];
          q[r] += w.counts(i) ? d * d : 0.f;
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < C; ++c) keep_narrow(raw[r][c]);
    row_sums<L>(q, red, turn);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Place<L, V, EVEN> w(c, lane, D);
      float ga[V], be[V];
      load_weight(gamma, w, 1.f, ga);
      load_weight(beta, w, 0.f, be);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t row = r0 + sub * R + r;
        if (row >= N) break;
        const float rstd = 1.f / sqrtf(q[r] * inv + eps);
        Chunk<T> y;
#pragma unroll
        for (int i = 0; i < V; ++i)
          y.v[i] = narrow<T>((widen(raw[r][c].v[i]) - mean[r]) * rstd * ga[i] + be[i]);
        store_chunk<L, EVEN>(Y + row * ldy, w, y);
        if (c == 0 && stats != nullptr && lane == 0) stats[row] = make_float2(mean[r], rstd);
      }
    }
  }
}

// dx row by row as above, and dgamma, dbeta summed in registers over the
// workgroup's rows; the groups of a workgroup are then added in LDS and each
// workgroup writes 2 D partial sums, so that the total has one fixed order.
// One workgroup of sixteen waves to a CU, each wave with R rows of x, dy and
// add in flight: 65,536 x 2,048 bfloat16 with add 215 us, 5.0 TB/s; 30,011 x 301
// float32 35 us, where vector instructions bound it as much as memory.
template <class T, class W, int L, int C, int R, bool EVEN>
__global__ __launch_bounds__(WIDE_GROUP) void norm_backward_kernel(
    const T* dY, int64_t lddy, const T* X, int64_t N, int D, int64_t ldx, const W* gamma,
    const float2* stats, const T* add, int64_t ldadd, T* dX, int64_t lddx, float* part) {
  constexpr int V = VEC<T>, ROWS = WIDE_GROUP / L * R;
  __shared__ float red[2][2 * R][WIDE_GROUP / WAVE];
  const int lane = threadIdx.x % L, sub = row_group<L>();
  float ga[V], dga[C][V], dbe[C][V];  // gamma is kept where it is one chunk
  load_weight(gamma, Place<L, V, EVEN>(0, lane, D), 1.f, ga);
#pragma unroll
  for (int c = 0; c < C; ++c) {
#pragma unroll
    for (int i = 0; i < V; ++i) dga[c][i] = dbe[c][i] = 0.f;
  }
  const float inv = 1.f / float(D);
  int turn = 0;
  for (int64_t r0 = int64_t(blockIdx.x) * ROWS; r0 < N; r0 += int64_t(gridDim.x) * ROWS) {
    Chunk<T> x[R][C], dy[R][C], ad[R][C];
    float2 st[R];
    float s[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = min(r0 + sub * R + r, N - 1);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Place<L, V, EVEN> w(c, lane, D);
        x[r][c] = load_chunk<L, EVEN>(X + row * ldx, w);
        dy[r][c] = load_chunk<L, EVEN>(dY + row * lddy, w);
        if (add != nullptr) ad[r][c] = load_chunk<L, EVEN>(add + row * ldadd, w);
        else ad[r][c] = Chunk<T>{};
      }
      st[r] = stats[row];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float live = r0 + sub * R + r < N ? 1.f : 0.f;
      s[r] = s[R + r] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Place<L, V, EVEN> w(c, lane, D);
        if (C > 1) load_weight(gamma, w, 1.f, ga);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float h = (widen(x[r][c].v[i]) - st[r].x) * st[r].y;
          // what does not count is a zero
          const float d = EVEN || w.counts(i) ? widen(dy[r][c].v[i]) : 0.f, g = d * ga[i];
          if (live != 0.f) {
            dga[c][i] += d * h;
            dbe[c][i] += d;
          }
          s[r] += g;
          s[R + r] += g * h;
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        keep_narrow(x[r][c]);
        keep_narrow(dy[r][c]);
      }
    row_sums<L>(s, red, turn);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = r0 + sub * R + r;
      if (row >= N) break;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Place<L, V, EVEN> w(c, lane, D);
        if (C > 1) load_weight(gamma, w, 1.f, ga);
        Chunk<T> out;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float h = (widen(x[r][c].v[i]) - st[r].x) * st[r].y;
          const float g = widen(dy[r][c].v[i]) * ga[i];
          float d = st[r].y * (g - s[r] * inv - h * (s[R + r] * inv));
          if (add != nullptr) d += widen(ad[r][c].v[i]);
          out.v[i] = narrow<T>(d);
        }
        store_chunk<L, EVEN>(dX + row * lddx, w, out);
      }
    }
  }
  if (part == nullptr) return;
  // groups of lanes of a wave, then the waves that hold the same features in order
  constexpr int S = L < WAVE ? WAVE : L, GROUPS = WIDE_GROUP / S;
  if (L < WAVE) {
#pragma unroll
    for (int d = L; d < WAVE; d *= 2)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        dga[0][i] += __shfl_xor(dga[0][i], d, WAVE);
        dbe[0][i] += __shfl_xor(dbe[0][i], d, WAVE);
      }
  }
  __shared__ float sums[GROUPS > 1 ? 2 * L * C * V : 1];
  const int group = threadIdx.x / S;
  for (int r = 0; r < GROUPS; ++r) {
    if (GROUPS > 1) __syncthreads();
    if (group != r || threadIdx.x % S >= L) continue;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Place<L, V, EVEN> w(c, lane, D);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!w.counts(i)) continue;
        const int f = w.at + i;
        float a = dga[c][i], b = dbe[c][i];
        if (GROUPS > 1) {
          if (r > 0) {
            a += sums[f];
            b += sums[L * C * V + f];
          }
          sums[f] = a;
          sums[L * C * V + f] = b;
        }
        if (r == GROUPS - 1) {
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
  if (col < 2 * D) {
#pragma unroll 16
    for (int64_t i = r; i < rows; i += 16) s += part[i * 2 * D + col];
  }
  sums[r][c] = s;
  __syncthreads();
  if (r != 0 || col >= 2 * D) return;
  for (int i = 1; i < 16; ++i) s += sums[i][c];
  W* out = col < D ? dgamma : dbeta;
  if (out != nullptr) out[col < D ? col : col - D] = narrow<W>(s);
}

// Rows too wide for registers (above 16,384 features; L = a workgroup a row),
// or less than 16 bytes (L = 1): read once for each sum, element by element.
template <int L>
__device__ __forceinline__ float other_sum(float s, float (*red)[1][GROUP / WAVE], int& turn) {
  float x[1] = {s};
  row_sums<L>(x, red, turn);
  return x[0];
}

template <class T, class W, int L>
__global__ __launch_bounds__(GROUP) void norm_other_kernel(const T* X, int64_t N, int64_t D,
                                                           int64_t ldx, const W* gamma,
                                                           const W* beta, float eps, T* Y,
                                                           int64_t ldy, float2* stats) {
  __shared__ float red[2][1][GROUP / WAVE];
  int turn = 0;
  const float inv = 1.f / float(D);
  const int lane = threadIdx.x % L, sub = threadIdx.x / L;
  constexpr int ROWS = GROUP / L;
  for (int64_t row = int64_t(blockIdx.x) * ROWS + sub; row < N; row += int64_t(gridDim.x) * ROWS) {
    const T* x = X + row * ldx;
    float s = 0.f;
    for (int64_t i = lane; i < D; i += L) s += widen(x[i]);
    const float mean = other_sum<L>(s, red, turn) * inv;
    s = 0.f;
    for (int64_t i = lane; i < D; i += L) {
      const float d = widen(x[i]) - mean;
      s += d * d;
    }
    const float rstd = 1.f / sqrtf(other_sum<L>(s, red, turn) * inv + eps);
    for (int64_t i = lane; i < D; i += L) {
      const float ga = gamma != nullptr ? widen(gamma[i]) : 1.f;
      const float be = beta != nullptr ? widen(beta[i]) : 0.f;
      Y[row * ldy + i] = narrow<T>((widen(x[i]) - mean) * rstd * ga + be);
    }
    if (stats != nullptr && lane == 0) stats[row] = make_float2(mean, rstd);
  }
}

template <class T, class W, int L>
__global__ __launch_bounds__(GROUP) void norm_other_backward_kernel(
    const T* dY, int64_t lddy, const T* X, int64_t N, int64_t D, int64_t ldx, const W* gamma,
    const float2* stats, const T* add, int64_t ldadd, T* dX, int64_t lddx) {
  __shared__ float red[2][2][GROUP / WAVE];
  int turn = 0;
  const float inv = 1.f / float(D);
  const int lane = threadIdx.x % L, sub = threadIdx.x / L;
  constexpr int ROWS = GROUP / L;
  for (int64_t row = int64_t(blockIdx.x) * ROWS + sub; row < N; row += int64_t(gridDim.x) * ROWS) {
    const T* x = X + row * ldx;
    const T* dy = dY + row * lddy;
    const float2 st = stats[row];
    float sums[2] = {0.f, 0.f};
    for (int64_t i = lane; i < D; i += L) {
      const float g = widen(dy[i]) * (gamma != nullptr ? widen(gamma[i]) : 1.f);
      sums[0] += g;
      sums[1] += g * ((widen(x[i]) - st.x) * st.y);
    }
    row_sums<L>(sums, red, turn);
    const float s = sums[0] * inv, sh = sums[1] * inv;
    for (int64_t i = lane; i < D; i += L) {
      const float g = widen(dy[i]) * (gamma != nullptr ? widen(gamma[i]) : 1.f);
      float d = st.y * (g - s - (widen(x[i]) - st.x) * st.y * sh);
      if (add != nullptr) d += widen(add[row * ldadd + i]);
      dX[row * lddx + i] = narrow<T>(d);
    }
  }
}

// Their partial sums of dgamma and dbeta, before dX (which may be dY): 64
// features of every gridDim.y-th four rows.
template <class T>
__global__ __launch_bounds__(GROUP) void norm_other_weight_kernel(
    const T* dY, int64_t lddy, const T* X, int64_t N, int64_t D, int64_t ldx, const float2* stats,
    float* part) {
  __shared__ float sums[2][4][WAVE];
  const int c = threadIdx.x % WAVE, r = threadIdx.x / WAVE;
  const int64_t f = int64_t(blockIdx.x) * WAVE + c;
  float a = 0.f, b = 0.f;
  if (f < D)
    for (int64_t row = int64_t(blockIdx.y) * 4 + r; row < N; row += int64_t(gridDim.y) * 4) {
      const float g = widen(dY[row * lddy + f]);
      a += g * ((widen(X[row * ldx + f]) - stats[row].x) * stats[row].y);
      b += g;
    }
  sums[0][r][c] = a;
  sums[1][r][c] = b;
  __syncthreads();
  if (r != 0 || f >= D) return;
  for (int i = 1; i < 4; ++i) {
    a += sums[0][i][c];
    b += sums[1][i][c];
  }
  part[int64_t(blockIdx.y) * 2 * D + f] = a;
  part[int64_t(blockIdx.y) * 2 * D + D + f] = b;
}

struct Forward {
  // rows of 513 to 1,024 chunks: 512 lanes x 2 (16,384 x 8,192 bfloat16: 101 us, 137 of 1,024 x 1)
  static constexpr int WIDEST = 1024;
  const void* X;
  int64_t N, D, ldx;
  const void *gamma, *beta;
  float eps;
  void* Y;
  int64_t ldy;
  float2* stats;
  hipStream_t stream;

  template <class T, class W, int L, int C, bool EVEN>
  void run() const {
    constexpr int R = C == 1 ? 4 : 4 / C, THREADS = L > GROUP ? L : GROUP;
    const int64_t grid = std::min<int64_t>(ceil_div(N, int64_t(THREADS / L * R)), 1 << 16);
    norm_kernel<T, W, L, C, R, EVEN><<<dim3(unsigned(grid)), dim3(THREADS), 0, stream>>>(
        static_cast<const T*>(X), N, int(D), ldx, static_cast<const W*>(gamma),
        static_cast<const W*>(beta), eps, static_cast<T*>(Y), ldy, stats);
  }
  template <class T, class W, int L>
  void other() const {
    const int64_t grid = std::min<int64_t>(ceil_div(N, int64_t(GROUP / L)), 8192);
    norm_other_kernel<T, W, L><<<dim3(unsigned(grid)), dim3(GROUP), 0, stream>>>(
        static_cast<const T*>(X), N, D, ldx, static_cast<const W*>(gamma),
        static_cast<const W*>(beta), eps, static_cast<T*>(Y), ldy, stats);
  }
};

int64_t norm_parts(int64_t N) { return std::min<int64_t>(N, PARTS); }

struct Backward {
  // and 1,024 lanes x 1 here (212 us, 289 of 512 x 2)
  static constexpr int WIDEST = 2048;
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

  template <class T, class W, int L, int C, bool EVEN>
  void run() const {
    constexpr int R = C == 1 ? 2 : 1;  // as many rows as fit 128 registers a lane
    const int64_t grid = std::min<int64_t>(ceil_div(N, int64_t(WIDE_GROUP / L * R)), PARTS);
    const bool weights = dgamma != nullptr || dbeta != nullptr;
    norm_backward_kernel<T, W, L, C, R, EVEN>
        <<<dim3(unsigned(grid)), dim3(WIDE_GROUP), 0, stream>>>(
            static_cast<const T*>(dY), lddy, static_cast<const T*>(X), N, int(D), ldx,
            static_cast<const W*>(gamma), stats, static_cast<const T*>(add), ldadd,
            static_cast<T*>(dX), lddx, weights ? part : nullptr);
    FD_LAUNCH_CHECK();
    if (weights) reduce<W>(grid);
  }
  template <class T, class W, int L>
  void other() const {
    if (dgamma != nullptr || dbeta != nullptr) {
      const int64_t parts = norm_parts(ceil_div(N, int64_t(4)));
      norm_other_weight_kernel<T>
          <<<dim3(unsigned(ceil_div(D, WAVE)), unsigned(parts)), dim3(GROUP), 0, stream>>>(
              static_cast<const T*>(dY), lddy, static_cast<const T*>(X), N, D, ldx, stats, part);
      FD_LAUNCH_CHECK();
      reduce<W>(parts);
      FD_LAUNCH_CHECK();
    }
    const int64_t grid = std::min<int64_t>(ceil_div(N, int64_t(GROUP / L)), 8192);
    norm_other_backward_kernel<T, W, L><<<dim3(unsigned(grid)), dim3(GROUP), 0, stream>>>(
        static_cast<const T*>(dY), lddy, static_cast<const T*>(X), N, D, ldx,
        static_cast<const W*>(gamma), stats, static_cast<const T*>(add), ldadd,
        static_cast<T*>(dX), lddx);
  }
  template <class W>
  void reduce(int64_t rows) const {
    norm_reduce_kernel<W><<<dim3(unsigned(ceil_div(2 * D, 16))), dim3(GROUP), 0, stream>>>(
        part, rows, D, static_cast<W*>(dgamma), static_cast<W*>(dbeta));
  }
};

// The narrowest group of lanes that holds a row: 16 lanes x 1 chunk up to
// 1,024 lanes x 16 elements (more would spill).
template <class T, class W, bool EVEN, class Call>
void by_width(const Call& call) {
  const int64_t chunks = ceil_div(call.D, VEC<T>);
  if (chunks <= 16) call.template run<T, W, 16, 1, EVEN>();
  else if (chunks <= 64) call.template run<T, W, 64, 1, EVEN>();
  else if (chunks <= 128) call.template run<T, W, 64, 2, EVEN>();
  else if (chunks <= 256) call.template run<T, W, 256, 1, EVEN>();
  else if (chunks <= 512) call.template run<T, W, 512, 1, EVEN>();
  else if (chunks <= 1024) call.template run<T, W, Call::WIDEST / 2, 2048 / Call::WIDEST, EVEN>();
  else if (chunks <= 2048) call.template run<T, W, 1024, 2, EVEN>();
  else if (chunks <= 16384 / VEC<T>) call.template run<T, W, 1024, 16 / VEC<T>, EVEN>();
  else call.template other<T, W, GROUP>();
  FD_LAUNCH_CHECK();
}
template <class T, class W, class Call>
void by_width(const Call& call) {
  if (call.D < VEC<T>) call.template other<T, W, 1>();  // not a chunk
  else if (call.D % VEC<T> == 0) by_width<T, W, true>(call);
  else by_width<T, W, false>(call);
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
