// AdamW over many tensors in few launches, states in 32 or 8 bits.
#include <algorithm>
#include <cmath>
#include <limits>

#include "fd_guard.hpp"
#include "net_common.hpp"

namespace fd {
namespace net {
namespace {

constexpr int BLOCK = 256;      // elements that share a scale, and threads of a workgroup
constexpr int CHUNK = 4096;     // elements of a workgroup
constexpr int64_t MAX_GROUPS = int64_t(1) << 23;  // workgroups of a launch
constexpr float E4M3_TOP = 448.f;
constexpr float E4M3_LEAST = 0x1p-9f;
constexpr float LEAST_TOP = 0x1p-100f;  // a block below this is stored as zeros

struct Tensor {
  float* p;
  const void* g;
  void* m;
  void* v;
  bf16* copy;
  int64_t n;
  int32_t gt;
  float keep;      // 1 - lr wd
};
struct ScaledTensor : Tensor {  // of 8-bit states
  float *ms, *vs;
};
struct Step {
  float b1, nb1, b2, nb2, rate, root, eps, gscale;
  uint32_t seed;  // of unbiased rounding: the step's
};
// The tensors of a launch travel in its arguments, of which there are 4 KB: a launch
// less is 5 to 7 us of a step (60 tensors, 14.9 million elements: 100 us in two, 92 in one).
template <class E, int COUNT>
struct Table {
  E t[COUNT];
  uint32_t first[COUNT + 1];  // a tensor's first workgroup
  int32_t count = 0;
};
using PlainTable = Table<Tensor, 64>;
using ScaledTable = Table<ScaledTensor, 48>;
static_assert(sizeof(PlainTable) + sizeof(Step) <= 4096 && sizeof(ScaledTable) + sizeof(Step) <= 4096,
              "a launch's arguments");

// The tensor of a workgroup: the last one whose first workgroup is not after it.
template <class TB>
__device__ __forceinline__ int find_tensor(const TB& tb, uint32_t wg) {
  int lo = 0, hi = tb.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (tb.first[mid] <= wg) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ void load_grad(const Tensor& t, int64_t at, int valid, float* g) {
  if (t.gt == FD_F32)
    load_wide<4>(static_cast<const float*>(t.g) + at, valid, g);
  else
    load_wide<4>(static_cast<const bf16*>(t.g) + at, valid, g);
}

// The moments and the update of one element, in the order that the formulas
// are written and without contraction: which of two neighbouring 8-bit values a
// moment rounds to then does not depend on the compiler.
__device__ __forceinline__ void update(const Step& s, float keep, float g, float& p, float& m,
                                       float& v, float& r) {
#pragma clang fp contract(off)
  g = g * s.gscale;
  m = s.b1 * m + s.nb1 * g;
  v = s.b2 * v + s.nb2 * (g * g);
  r = sqrtf(v);
  p = p * keep - s.rate * m / (r * s.root + s.eps);
}

// Bound by memory, 24 bytes an element and the gradient (28 in float32; 2 less and a
// copy's 2 more in bfloat16).  Four elements of a lane are one 16-byte access of each
// array; a lane asks for all its elements before it updates the first (107 -> 100 us for
// 14.9 million, 92 us and 4.5 TB/s in one launch).
__global__ __launch_bounds__(BLOCK) void adamw_kernel(PlainTable tb, Step s) {
  const int ti = find_tensor(tb, blockIdx.x);
  const Tensor& t = tb.t[ti];
  const int64_t base = int64_t(blockIdx.x - tb.first[ti]) * CHUNK;
  float* M = static_cast<float*>(t.m);
  float* V = static_cast<float*>(t.v);
  constexpr int EACH = CHUNK / (BLOCK * 4);
  float p[EACH][4], g[EACH][4], m[EACH][4], v[EACH][4], r;
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int64_t at = base + (j * BLOCK + int(threadIdx.x)) * 4;
    const int valid = int(max(int64_t(0), min(int64_t(4), t.n - at)));
    load_wide<4>(t.p + at, valid, p[j]);
    load_grad(t, at, valid, g[j]);
    load_wide<4>(M + at, valid, m[j]);
    load_wide<4>(V + at, valid, v[j]);
  }
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int64_t at = base + (j * BLOCK + int(threadIdx.x)) * 4;
    const int valid = int(max(int64_t(0), min(int64_t(4), t.n - at)));
#pragma unroll
    for (int i = 0; i < 4; ++i) update(s, t.keep, g[j][i], p[j][i], m[j][i], v[j][i], r);
    store_wide<4>(t.p + at, valid, p[j]);
    store_wide<4>(M + at, valid, m[j]);
    store_wide<4>(V + at, valid, v[j]);
    if (t.copy != nullptr) store_wide<4>(t.copy + at, valid, p[j]);
  }
}

__device__ __forceinline__ int load_e4m3(const unsigned char* q, int valid) {
  int w = 0;
  if (valid >= 4) {
    __builtin_memcpy(&w, q, 4);
  } else {
    for (int i = 0; i < valid; ++i) w |= int(q[i]) << (8 * i);
  }
  return w;
}

__device__ __forceinline__ void widen_e4m3(int w, float scale, float* out) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  out[0] = lo[0] * scale;
  out[1] = lo[1] * scale;
  out[2] = hi[0] * scale;
  out[3] = hi[1] * scale;
}

// 32 well mixed bits of a number and a seed: every element and step has its own,
// the same in every run.
__host__ __device__ inline uint32_t mix(uint64_t at, uint32_t seed) {
  uint32_t h = (uint32_t(at) * 0x9e3779b1u) ^ (uint32_t(at >> 32) * 0xddb3d743u) ^ seed;
  h ^= h >> 16;
  h *= 0xb504f333u;
  h ^= h >> 15;
  h *= 0xddb3d743u;
  return h ^ (h >> 16);
}

// |y| <= 448 to one of the e4m3 values around it, up where `bits` as a fraction of one is
// below the chance that makes the value's mean y; for a root, its square's mean y^2.
// An e4m3 value is a float32 with 20 zero bits at the end, once 2^-6 is added to those below it.
template <bool ROOT>
__device__ __forceinline__ float round_e4m3(float y, uint32_t bits) {
  const float a = fabsf(y), shift = a < 0x1p-6f ? 0x1p-6f : 0.f;
  const uint32_t w = __builtin_bit_cast(uint32_t, a + shift) & 0xfff00000u;
  const float lo = __builtin_bit_cast(float, w) - shift;
  const float hi = __builtin_bit_cast(float, w + 0x100000u) - shift;
  float want = a - lo, gap = hi - lo;
  if (ROOT) {
    want *= a + lo;
    gap *= hi + lo;
  }
  const float u = float(bits >> 8) * 0x1p-24f;
  return copysignf(fminf(u * gap < want ? hi : lo, E4M3_TOP), y);
}

// Four values of a block whose largest finite magnitude is found over the wave;
// returns the block's scale.  bits: four words for UNBIASED rounding.
template <bool ROOT, bool UNBIASED>
__device__ __forceinline__ float narrow_e4m3(const float* x, unsigned char* q, int valid,
                                             const uint32_t* bits) {
#pragma clang fp contract(off)
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = fabsf(x[i]);
    if (i < valid && a < INFINITY) top = fmaxf(top, a);
  }
  top = wave_max(top);
  if (top < LEAST_TOP) top = 0.f;
  const float inv = top > 0.f ? (1.0f / top) * E4M3_TOP : 0.f;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = x[i] * inv;
    if (ROOT && x[i] > 0.f && inv > 0.f) y[i] = fmaxf(y[i], E4M3_LEAST);
    if (UNBIASED) y[i] = round_e4m3<ROOT>(y[i], bits[i]);
    if (!(fabsf(x[i]) < INFINITY)) y[i] = NAN;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  if (valid >= 4) {
    __builtin_memcpy(q, &w, 4);
  } else {
    for (int i = 0; i < valid; ++i) q[i] = static_cast<unsigned char>(w >> (8 * i));
  }
  return top * (1.0f / E4M3_TOP);
}

// The 8-bit form: one wave takes the 256 elements that share a scale, so that
// the new scale is a maximum over its lanes.  12 bytes an element, the gradient and the copy:
// 152 million elements in 468 us, 5.2 TB/s; with unbiased rounding, whose vector instructions
// bound it, in 575.
template <bool UNBIASED>
__global__ __launch_bounds__(BLOCK) void adamw_e4m3_kernel(ScaledTable tb, Step s) {
  const int ti = find_tensor(tb, blockIdx.x);
  const ScaledTensor& t = tb.t[ti];
  const int64_t base = int64_t(blockIdx.x - tb.first[ti]) * CHUNK;
  unsigned char* M = static_cast<unsigned char*>(t.m);
  unsigned char* V = static_cast<unsigned char*>(t.v);
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
  constexpr int EACH = CHUNK / (BLOCK * 4);
  float p[EACH][4], g[EACH][4], ms[EACH], vs[EACH];
  int qm[EACH], qv[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int64_t block = base + (j * (BLOCK / WAVE) + wave) * BLOCK, at = block + lane * 4;
    const int valid = int(max(int64_t(0), min(int64_t(4), t.n - at)));
    load_wide<4>(t.p + at, valid, p[j]);
    load_grad(t, at, valid, g[j]);
    qm[j] = load_e4m3(M + at, valid);
    qv[j] = load_e4m3(V + at, valid);
    ms[j] = block < t.n ? t.ms[block / BLOCK] : 0.f;
    vs[j] = block < t.n ? t.vs[block / BLOCK] : 0.f;
  }
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int64_t block = base + (j * (BLOCK / WAVE) + wave) * BLOCK;
    if (block >= t.n) break;  // the whole wave
    const int64_t at = block + lane * 4;
    const int valid = int(max(int64_t(0), min(int64_t(4), t.n - at)));
    float m[4], v[4], r[4];
    widen_e4m3(qm[j], ms[j], m);
    widen_e4m3(qv[j], vs[j], r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = r[i] * r[i];
      update(s, t.keep, g[j][i], p[j][i], m[i], v[i], r[i]);
    }
    store_wide<4>(t.p + at, valid, p[j]);
    if (t.copy != nullptr) store_wide<4>(t.copy + at, valid, p[j]);
    uint32_t mb[4], rb[4];
    if (UNBIASED)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mb[i] = mix(uint64_t(at + i), s.seed);
        rb[i] = mix(mb[i], s.seed);
      }
    const float m1 = narrow_e4m3<false, UNBIASED>(m, M + at, valid, mb);
    const float r1 = narrow_e4m3<true, UNBIASED>(r, V + at, valid, rb);
    if (lane == 0) {
      t.ms[block / BLOCK] = m1;
      t.vs[block / BLOCK] = r1;
    }
  }
}

void set_scales(Tensor&, const fd_adamw_tensor&) {}
void set_scales(ScaledTensor& d, const fd_adamw_tensor& t) {
  d.ms = t.m_scale;
  d.vs = t.v_scale;
}

// A launch for each table of tensors, or 2^23 workgroups (2^31 threads).
template <class TB>
void run(void (*kernel)(TB, Step), const fd_adamw_tensor* tensors, int64_t count,
         const fd_adamw_opts& o, const Step& s, hipStream_t st) {
  constexpr int ROOM = int(sizeof(TB::t) / sizeof(TB::t[0]));
  TB tb{};
  int64_t groups = 0;
  auto flush = [&] {
    if (tb.count == 0) return;
    tb.first[tb.count] = uint32_t(groups);
    kernel<<<dim3(unsigned(groups)), dim3(BLOCK), 0, st>>>(tb, s);
    FD_LAUNCH_CHECK();
    tb.count = 0;
    groups = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const fd_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    const int64_t need = ceil_div(t.n, CHUNK);
    if (tb.count == ROOM || groups + need > MAX_GROUPS) flush();
    auto& d = tb.t[tb.count];
    d.p = t.p;
    d.g = t.g;
    d.m = t.m;
    d.v = t.v;
    d.copy = static_cast<bf16*>(t.copy);
    d.n = t.n;
    d.gt = t.gt;
    d.keep = float(1.0 - o.lr * o.weight_decay * double(t.decay));
    set_scales(d, t);
    tb.first[tb.count] = uint32_t(groups);
    ++tb.count;
    groups += need;
  }
  flush();
}

}  // namespace
}  // namespace net
}  // namespace fd

using namespace fd;
using namespace fd::net;

extern "C" {

void fd_adamw_default_opts(fd_adamw_opts* o) {
  if (o == nullptr) return;
  *o = fd_adamw_opts{};
  o->lr = 1e-3;
  o->beta1 = 0.9;
  o->beta2 = 0.999;
  o->eps = 1e-8;
  o->weight_decay = 0.01;
  o->grad_scale = 1.0;
  o->step = 1;
  o->state_bits = 32;
}

fd_status fd_adamw_step(const fd_adamw_tensor* tensors, int64_t count, const fd_adamw_opts* opts,
                        void* stream) {
  return guarded([&] {
    FD_REQUIRE(count >= 0 && (count == 0 || tensors != nullptr), FD_ERR_INVALID_ARG,
               "bad tensor list");
    fd_adamw_opts o;
    fd_adamw_default_opts(&o);
    if (opts != nullptr) o = *opts;
    FD_REQUIRE(o.state_bits == 32 || o.state_bits == 8, FD_ERR_UNSUPPORTED,
               "state_bits must be 32 or 8");
    FD_REQUIRE(o.step >= 1, FD_ERR_INVALID_ARG, "step must be >= 1");
    FD_REQUIRE(o.beta1 >= 0 && o.beta1 < 1 && o.beta2 >= 0 && o.beta2 < 1, FD_ERR_INVALID_ARG,
               "beta1 and beta2 must be in [0, 1)");
    FD_REQUIRE(std::isfinite(o.lr) && o.eps >= 0 && std::isfinite(o.eps) &&
                   std::isfinite(o.weight_decay) && std::isfinite(o.grad_scale),
               FD_ERR_INVALID_ARG, "lr, eps, weight_decay and grad_scale must be finite, eps >= 0");
    const bool narrow_states = o.state_bits == 8;
    FD_REQUIRE(o.rounding == FD_ROUND_NEAREST || o.rounding == FD_ROUND_UNBIASED,
               FD_ERR_INVALID_ARG, "unknown rounding");
    for (int64_t i = 0; i < count; ++i) {
      const fd_adamw_tensor& t = tensors[i];
      FD_REQUIRE(t.n >= 0 && t.n <= MAX_GROUPS * CHUNK, FD_ERR_INVALID_ARG, "tensor size out of range");
      if (t.n == 0) continue;
      check_dtype(t.gt, "gradient dtype");
      FD_REQUIRE(t.p != nullptr && t.g != nullptr && t.m != nullptr && t.v != nullptr,
                 FD_ERR_INVALID_ARG, "tensor with a NULL array");
      FD_REQUIRE(!narrow_states || (t.m_scale != nullptr && t.v_scale != nullptr),
                 FD_ERR_INVALID_ARG, "8-bit states need their scales");
      FD_REQUIRE(std::isfinite(t.decay), FD_ERR_INVALID_ARG, "decay must be finite");
      check_element_aligned(t.p, FD_F32, "p");
      check_element_aligned(t.g, t.gt, "g");
      if (t.copy != nullptr) check_element_aligned(t.copy, FD_BF16, "copy");
      check_element_aligned(narrow_states ? t.m_scale : t.m, FD_F32, "m");
      check_element_aligned(narrow_states ? t.v_scale : t.v, FD_F32, "v");
    }
    Step s;
    s.b1 = float(o.beta1);
    s.nb1 = float(1.0 - o.beta1);
    s.b2 = float(o.beta2);
    s.nb2 = float(1.0 - o.beta2);
    s.rate = float(o.lr / (1.0 - std::pow(o.beta1, double(o.step))));
    s.root = float(1.0 / std::sqrt(1.0 - std::pow(o.beta2, double(o.step))));
    // an eps that float32 would round to zero still keeps 0 / (0 + eps) at zero
    s.eps = o.eps > 0 ? std::max(float(o.eps), std::numeric_limits<float>::min()) : 0.f;
    s.gscale = float(o.grad_scale);
    s.seed = mix(uint64_t(o.step), 0x6a09e667u);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (narrow_states)
      run<ScaledTable>(o.rounding == FD_ROUND_UNBIASED ? adamw_e4m3_kernel<true> : adamw_e4m3_kernel<false>,
                       tensors, count, o, s, st);
    else
      run<PlainTable>(adamw_kernel, tensors, count, o, s, st);
  });
}

}  // extern "C"
