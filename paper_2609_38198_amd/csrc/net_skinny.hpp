// Products of few rows with a weight matrix, C[n][f] = sum_k X(n, k) W(f, k):
// the gated block at one point or a small batch, where the time is the
// weights' way from memory.
#pragma once

#include "net_gemm.hpp"

namespace fd {
namespace net {

constexpr int SKINNY_WAVES = 16;  // waves x 16-row blocks of a workgroup at most

struct SkinnyArgs {
  const void* x;            // n rows
  const void *w, *up;       // F x K each (up: the gate product's second matrix)
  int64_t ldx, ldw, n, F, K;
  const void *b, *bu;       // biases or NULL
  const void* R;            // added, or NULL
  int64_t ldr;
  void* out;
  int64_t ldo;
  int64_t xplane, plane;    // elements between planes of x, out
};

// A workgroup makes 16 columns of C for NB x 16 rows; its W waves share the
// columns and take every W-th stretch of k, whose weights go straight from
// memory to the matrix operand: 16 rows x 64 k (float32: 32) of each
// matrix in flight at once, every weight read once and by one wave.  The sum over the waves, in their
// order, is in LDS.  1 x 1024 -> 4096 -> 1024 in bfloat16 moves 17 MB in 5.4 us and 8 MB in 7.8 us:
// latency, of one trip to memory for each of the 64 workgroups' waves, more than bandwidth.
//
// HP: the planes of H in bfloat16, which the first product writes and the second reads.
template <class T, int HP, int NB, int W, bool GATED, int ACT>
__global__ __launch_bounds__(W * WAVE) void skinny_kernel(SkinnyArgs p) {
  constexpr int MATS = GATED ? 2 : 1;
  constexpr int V = VEC<T>, KC = 8 * V;  // k of a step: two loads of 16 bytes by four lane groups
  __shared__ float red[W][MATS][NB][16][17];
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
  const int64_t f0 = int64_t(blockIdx.x) * 16;
  const int64_t f = min(f0 + lane % 16, p.F - 1);
  const T* w[MATS];
  w[0] = static_cast<const T*>(p.w) + f * p.ldw;
  if (GATED) w[MATS - 1] = static_cast<const T*>(p.up) + f * p.ldw;
  constexpr int XP = GATED ? 1 : HP;
  const T* x[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
    x[i] = static_cast<const T*>(p.x) + min(int64_t(i * 16 + lane % 16), p.n - 1) * p.ldx;
  floatx4 acc[MATS][NB];
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int i = 0; i < NB; ++i) acc[m][i] = floatx4{0.f, 0.f, 0.f, 0.f};

  struct Chunk {
    T v[V];
  };
  auto load = [](const T* q, int64_t left) {
    Chunk c;
    if (left >= V) {
      __builtin_memcpy(&c, q, 16);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) c.v[e] = e < left ? q[e] : T(0.f);
    }
    return c;
  };
  auto step = [&](int64_t k0, bool whole) {
    // lane group l / 16 has k = k0 + 2 V (l / 16) + V j + 0 .. V - 1
    Chunk cw[MATS][2], cx[NB][2][XP];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t k = k0 + (lane / 16) * 2 * V + j * V;
      const int64_t left = whole ? V : p.K - k;
#pragma unroll
      for (int m = 0; m < MATS; ++m) cw[m][j] = load(w[m] + k, left);
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int q = 0; q < XP; ++q) cx[i][j][q] = load(x[i] + q * p.xplane + k, left);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int m = 0; m < MATS; ++m)
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int q = XP - 1; q >= 0; --q)
              acc[m][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, cw[m][j]), __builtin_bit_cast(bf16x8, cx[i][j][q]),
                  acc[m][i], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
              acc[m][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(cw[m][j].v[e], cx[i][j][0].v[e],
                                                               acc[m][i], 0, 0, 0);
          }
        }
  };
  int64_t k = wave * KC;
  for (; k + KC <= p.K; k += W * KC) step(k, true);
  if (k < p.K) step(k, false);

#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[wave][m][i][(lane / 16) * 4 + e][lane % 16] = acc[m][i][e];
  __syncthreads();
  for (int at = threadIdx.x; at < NB * 256; at += W * WAVE) {
    const int c = at % 16, r = at / 16 % 16, i = at / 256;
    const int64_t row = i * 16 + r, col = f0 + c;
    if (row >= p.n || col >= p.F) continue;
    float s[MATS] = {};
    for (int v = 0; v < W; ++v)
#pragma unroll
      for (int m = 0; m < MATS; ++m) s[m] += red[v][m][i][c][r];
    if (p.b != nullptr) s[0] += widen(static_cast<const T*>(p.b)[col]);
    if (GATED) {
      if (p.bu != nullptr) s[MATS - 1] += widen(static_cast<const T*>(p.bu)[col]);
      s[0] = activate<ACT, T>(s[0]).value * s[MATS - 1];
    }
    if (p.R != nullptr) s[0] += widen(static_cast<const T*>(p.R)[row * p.ldr + col]);
    T* out = static_cast<T*>(p.out) + row * p.ldo + col;
    if constexpr (GATED && HP == 2) {
      bf16 v[2];
      to_planes<2>(s[0], v);
      out[0] = v[0];
      out[p.plane] = v[1];
    } else {
      *out = narrow<T>(s[0]);
    }
  }
}

// As many waves as have a stretch of k each (a power of two).
template <class T, int HP, int NB, bool GATED, int ACT>
void launch_skinny_blocks(const SkinnyArgs& p, hipStream_t stream) {
  const int64_t stretches = ceil_div(p.K, 8 * VEC<T>);
  const dim3 grid(unsigned(ceil_div(p.F, int64_t(16))));
  if (SKINNY_WAVES / NB >= 16 && stretches > 8) {
    constexpr int W = SKINNY_WAVES / NB < 16 ? 1 : 16;
    skinny_kernel<T, HP, NB, W, GATED, ACT><<<grid, dim3(W * WAVE), 0, stream>>>(p);
  } else if (SKINNY_WAVES / NB >= 8 && stretches > 4) {
    constexpr int W = SKINNY_WAVES / NB < 8 ? 1 : 8;
    skinny_kernel<T, HP, NB, W, GATED, ACT><<<grid, dim3(W * WAVE), 0, stream>>>(p);
  } else {
    skinny_kernel<T, HP, NB, 4, GATED, ACT><<<grid, dim3(4 * WAVE), 0, stream>>>(p);
  }
  FD_LAUNCH_CHECK();
}

template <class T, int HP, bool GATED, int ACT>
void launch_skinny(const SkinnyArgs& p, hipStream_t stream) {
  if (p.n <= 16) launch_skinny_blocks<T, HP, 1, GATED, ACT>(p, stream);
  else if (p.n <= 32) launch_skinny_blocks<T, HP, 2, GATED, ACT>(p, stream);
  else launch_skinny_blocks<T, HP, 4, GATED, ACT>(p, stream);
}

}  // namespace net
}  // namespace fd
