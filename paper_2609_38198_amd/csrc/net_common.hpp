// Shared device and host helpers of the parametric extension's operators
// (layer norm, gated block, AdamW).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fd_internal.hpp"

namespace fd {
namespace net {

using bf16 = __bf16;
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int WAVE = 64;


// Elements of type T in 16 bytes, the widest load of a lane.
template <class T>
constexpr int VEC = 16 / int(sizeof(T));

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16 x) { return float(x); }
template <class T>
__device__ __forceinline__ T narrow(float x) {  // to nearest, ties to even
  return static_cast<T>(x);
}

// N elements at p (aligned to one element only: global memory takes wide
// accesses at any address) into float32; those from `valid` on read as zero
// and are not touched.
template <int N, class T>
__device__ __forceinline__ void load_wide(const T* __restrict__ p, int valid, float* out) {
  if (valid >= N) {
    T v[N];
    __builtin_memcpy(v, p, sizeof(v));
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = widen(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = i < valid ? widen(p[i]) : 0.f;
  }
}

template <int N, class T>
__device__ __forceinline__ void store_wide(T* __restrict__ p, int valid, const float* in) {
  if (valid >= N) {
    T v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = narrow<T>(in[i]);
    __builtin_memcpy(p, v, sizeof(v));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < valid) p[i] = narrow<T>(in[i]);
  }
}

// Sum over groups of L consecutive lanes (L a power of two), in every lane.
template <int L>
__device__ __forceinline__ float lane_sum(float x) {
#pragma unroll
  for (int d = L / 2; d > 0; d >>= 1) x += __shfl_xor(x, d, WAVE);
  return x;
}

// Maximum over the wave, by data-parallel moves: within rows of 16 lanes, then
// from row to row into lane 63.
__device__ __forceinline__ float wave_max(float x) {
  auto step = [&](auto moved) { x = fmaxf(x, __builtin_bit_cast(float, moved)); };
  const auto bits = [&] { return __builtin_bit_cast(int, x); };
  step(__builtin_amdgcn_update_dpp(bits(), bits(), 0x111, 0xf, 0xf, false));  // row_shr:1
  step(__builtin_amdgcn_update_dpp(bits(), bits(), 0x112, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(bits(), bits(), 0x114, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(bits(), bits(), 0x118, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(bits(), bits(), 0x142, 0xa, 0xf, false));  // row_bcast:15
  step(__builtin_amdgcn_update_dpp(bits(), bits(), 0x143, 0xc, 0xf, false));  // row_bcast:31
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(bits(), WAVE - 1));
}

// A launch holds fewer than 2^32 threads; one of more runs what is left over them
// alone, without an error.
inline void check_launch(int64_t groups, int64_t threads) {
  FD_REQUIRE(groups < (int64_t(1) << 32) / threads, FD_ERR_UNSUPPORTED,
             "problem too large for one launch");
}

// Checks shared by the entry points.
inline void check_dtype(int t, const char* what) {
  FD_REQUIRE(t == FD_F32 || t == FD_BF16, FD_ERR_INVALID_ARG, std::string("unknown ") + what);
}
inline size_t type_size(int t) { return t == FD_F32 ? 4 : 2; }
constexpr int64_t MAX_ROWS = int64_t(1) << 30;
constexpr int64_t MAX_WIDTH = int64_t(1) << 20;
inline void check_element_aligned(const void* p, int t, const char* what) {
  FD_REQUIRE((reinterpret_cast<uintptr_t>(p) & (type_size(t) - 1)) == 0, FD_ERR_INVALID_ARG,
             std::string(what) + " is not aligned to its elements");
}

}  // namespace net
}  // namespace fd
