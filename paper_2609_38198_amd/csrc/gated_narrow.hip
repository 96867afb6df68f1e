// The gated block's narrow forward pass.
#include <type_traits>
#include <utility>

#include "net_gemm.hpp"
#include "net_narrow.hpp"

namespace fd {
namespace net {
namespace {

// f(0), f(1), ... with constants: an array that it indexes stays in registers,
// however long its body.
template <int... I, class F>
__device__ __forceinline__ void for_each_of(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void for_each_of(F f) {
  for_each_of(std::make_integer_sequence<int, N>{}, f);
}

// Eight values as they are in memory: nothing waits for them until they are widened.
// `room`: how many there are to the matrix's last one; what lies past the row's
// end is another row's or padding, and is put to zero on widening.
template <class T>
struct Eight {
  typedef T Vec __attribute__((ext_vector_type(8)));
};
template <class T>
__device__ __forceinline__ typename Eight<T>::Vec load_eight(const T* p, int64_t room) {
  typename Eight<T>::Vec v;
  if (room >= 8) {
    __builtin_memcpy(&v, p, sizeof(v));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = T(0.f);
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < room) v[e] = p[e];
  }
  return v;
}

// A wave keeps 32 rows of X and of Y in registers and walks F by 32: G and U of
// a 32 x 32 block on the matrix unit, H in the accumulators' registers, and from there
// straight into the product with Wd.  An accumulator holds, of row l % 32,
// f = 8 (i / 4) + 4 (l / 32) + i % 4; the second product's order of f within a k
// step is free as long as Wd's operand has the same, so H needs no exchange between lanes.
// Nothing inner goes to memory: 30,011 x 30 -> 512 -> 64 in float32 takes 42 us,
// 85 with tiles that write H and read it; 1,000,000 x 30 -> 256 -> 64 in bfloat16 184 us and
// 493.  Bound by the vector unit (activations, splitting into planes) about as
// much as by the matrix unit.  The NW waves of a workgroup share the weights, widened
// to planes on their way to LDS one step of F ahead; any alignment will do.
template <class T, int DP, int OP, int NW, int ACT, int HP>
__global__ __launch_bounds__(NW * WAVE, 2) void narrow_kernel(NarrowArgs p) {
  constexpr int PL = planes_of<T>, KS = DP / 16, OB = OP / 32, THREADS = NW * WAVE;
  // LDS rows of DP (32) values, 16 bytes more apart: eight rows' same chunk cover all banks
  constexpr int WP = DP + 8, VP = 32 + 8;
  constexpr int CHUNKS = 2 * 32 * DP / 8 + OP * 4, EACH = (CHUNKS + THREADS - 1) / THREADS;
  struct Buffer {
    bf16 w[PL][2][32][WP];  // gate, up
    bf16 d[PL][OP][VP];
    float bias[2][32];
  };
  __shared__ __align__(16) Buffer buf[2];
  const fd_gated_block& b = p.b;
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE, half = lane / 32;
  const int64_t m0 = (int64_t(blockIdx.x) * NW + wave) * 32, m = m0 + lane % 32;

  // The weights of 32 inner features, 8 values at a time: the first 8 DP of
  // CHUNKS are gate and up (row f, columns c on), the rest down (row o).
  struct Source {
    const T* p;
    int64_t step;  // elements to the next 32 features
    int64_t room;  // elements to the matrix's end
    int row, valid;  // gate, up: f within the step; valid values (down: less the step's f)
  };
  const int64_t steps = (b.F + 31) / 32;
  const int64_t f_first = steps * blockIdx.y / p.parts * 32;
  const int64_t f_last = min(steps * (blockIdx.y + 1) / p.parts * 32, b.F);
  Source src[EACH];
  for_each_of<EACH>([&](auto i) {
    const int q = threadIdx.x + i * THREADS;
    if (q < 8 * DP) {
      const int r = q % (4 * DP) / (DP / 8), c = q % (DP / 8) * 8;
      const T* w = static_cast<const T*>(q < 4 * DP ? b.Wg : b.Wu);
      src[i] = Source{w + (f_first + r) * b.ldwi + c, 32 * b.ldwi,
                      (b.F - 1 - f_first - r) * b.ldwi + b.D - c, r, int(b.D) - c};
    } else {
      const int r = (q - 8 * DP) / 4, c = (q - 8 * DP) % 4 * 8;
      const bool there = q < CHUNKS && r < b.O;
      src[i] = Source{static_cast<const T*>(b.Wd) + (there ? r : 0) * b.ldwd + f_first + c, 32,
                      there ? (b.O - 1 - r) * b.ldwd + b.F - f_first - c : 0, 0,
                      there ? c : 1 << 20};
    }
  });
  typename Eight<T>::Vec raw[EACH];
  T bias = T(0.f);
  auto fetch = [&](int64_t f0) {
    for_each_of<EACH>([&](auto i) {
      raw[i] = load_eight(src[i].p, src[i].room);
      src[i].p += src[i].step;
      src[i].room -= src[i].step;
    });
    if (threadIdx.x < 64) {
      const T* v = static_cast<const T*>(threadIdx.x < 32 ? b.bg : b.bu);
      const int64_t f = f0 + threadIdx.x % 32;
      bias = v != nullptr && f < b.F ? v[f] : T(0.f);
    }
  };
  auto put = [&](Buffer& to, int64_t f0) {
    const int left = int(min(b.F - f0, int64_t(32)));
    for_each_of<EACH>([&](auto i) {
      const int q = threadIdx.x + i * THREADS;
      const int valid = q < 8 * DP ? (src[i].row < left ? src[i].valid : 0) : left - src[i].valid;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < valid ? widen(T(raw[i][e])) : 0.f;
      if (q < 8 * DP)
        write_planes<PL>(&to.w[0][q / (4 * DP)][q % (4 * DP) / (DP / 8)][q % (DP / 8) * 8], 2 * 32 * WP, v);
      else if (q < CHUNKS)
        write_planes<PL>(&to.d[0][(q - 8 * DP) / 4][(q - 8 * DP) % 4 * 8], OP * VP, v);
    });
    if (threadIdx.x < 64) to.bias[threadIdx.x / 32][threadIdx.x % 32] = widen(bias);
  };
  using P = Pairs<PL, PL>;
  using Q = Pairs<HP, PL>;

  fetch(f_first);
  bf16x8 x[KS][PL];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    float v[8];
    const int k = s * 16 + half * 8;
    load_wide<8>(static_cast<const T*>(b.X) + min(m, b.N - 1) * b.ldx + k, int(b.D) - k, v);
    to_planes<PL>(v, x[s]);
  }
  floatx16 y[OB];
#pragma unroll
  for (int o = 0; o < OB; ++o)
#pragma unroll
    for (int e = 0; e < 16; ++e) y[o][e] = 0.f;
  put(buf[0], f_first);

  int cur = 0;
  for (int64_t f0 = f_first; f0 < f_last; f0 += 32, cur ^= 1) {
    __syncthreads();
    const Buffer& w = buf[cur];
    if (f0 + 32 < f_last) fetch(f0 + 32);
    floatx16 g, u, gl, ul;  // low: the smaller plane pairs' sums
#pragma unroll
    for (int e = 0; e < 16; ++e) g[e] = u[e] = gl[e] = ul[e] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      bf16x8 wg[PL], wu[PL];
#pragma unroll
      for (int q = 0; q < PL; ++q) {
        wg[q] = *reinterpret_cast<const bf16x8*>(&w.w[q][0][lane % 32][s * 16 + half * 8]);
        wu[q] = *reinterpret_cast<const bf16x8*>(&w.w[q][1][lane % 32][s * 16 + half * 8]);
      }
#pragma unroll
      for (int q = 0; q < P::COUNT; ++q) {
        floatx16 &tg = q + 1 == P::COUNT ? g : gl, &tu = q + 1 == P::COUNT ? u : ul;
        const bf16x8 xs = x[s][P::a(q)];
        tg = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wg[P::b(q)], xs, tg, 0, 0, 0);
        tu = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wu[P::b(q)], xs, tu, 0, 0, 0);
      }
    }
    if (PL > 1) {
      g += gl;
      u += ul;
    }
    // last, and all in the tiles' order: both make the same bits
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const floatx4 bg = *reinterpret_cast<const floatx4*>(&w.bias[0][8 * q + 4 * half]);
      const floatx4 bu = *reinterpret_cast<const floatx4*>(&w.bias[1][8 * q + 4 * half]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g[4 * q + e] += bg[e];
        u[4 * q + e] += bu[e];
      }
    }
    if (p.saved != nullptr && m0 < b.N) {
      char* block = saved_at<T>(p.saved, m0, f0, p.Fp);
      save16<T>(block, 0, lane, g);
      save16<T>(block, 1, lane, u);
    }
    // past F the weights and biases are zero, and so is H
    float h[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) h[e] = activate<ACT, T>(g[e]).value * u[e];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 hp[HP];
      to_planes<HP>(h + 8 * s, hp);
      bf16x8 wd[OB][PL];
#pragma unroll
      for (int o = 0; o < OB; ++o)
#pragma unroll
        for (int q = 0; q < PL; ++q) {
          const bf16* r = &w.d[q][o * 32 + lane % 32][s * 16 + 4 * half];
          const bf16x4 lo = *reinterpret_cast<const bf16x4*>(r), hi = *reinterpret_cast<const bf16x4*>(r + 8);
          wd[o][q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
#pragma unroll
      for (int q = 0; q < Q::COUNT; ++q)
#pragma unroll
        for (int o = 0; o < OB; ++o)
          y[o] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wd[o][Q::b(q)], hp[Q::a(q)], y[o], 0, 0, 0);
    }
    // the other buffer was last read before this step's barrier
    if (f0 + 32 < f_last) put(buf[cur ^ 1], f0 + 32);
  }

  if (m >= b.N) return;
#pragma unroll
  for (int o = 0; o < OB; ++o)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = o * 32 + 8 * q + 4 * half, valid = min(4, int(b.O) - col);
      if (valid <= 0) continue;
      float v[4], r[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = y[o][4 * q + e];
      if (p.parts > 1) {
        store_wide<4>(p.part + (blockIdx.y * b.N + m) * p.ldp + col, valid, v);
        continue;
      }
      if (b.bd != nullptr) {
        load_wide<4>(static_cast<const T*>(b.bd) + col, valid, r);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += r[e];
      }
      if (p.R != nullptr) {
        load_wide<4>(static_cast<const T*>(p.R) + m * p.ldr + col, valid, r);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += r[e];
      }
      store_wide<4>(static_cast<T*>(p.Y) + m * p.ldy + col, valid, v);
    }
}

template <class T, int DP, int OP, int ACT, int HP>
void launch(const NarrowArgs& p, hipStream_t stream) {
  constexpr int NW = NARROW_ROWS / 32;
  const dim3 grid(unsigned(ceil_div(p.b.N, NARROW_ROWS)), unsigned(p.parts));
  narrow_kernel<T, DP, OP, NW, ACT, HP><<<grid, dim3(NW * WAVE), 0, stream>>>(p);
  FD_LAUNCH_CHECK();
}

template <class T, int ACT, int HP>
void launch_narrow(const NarrowArgs& p, hipStream_t stream) {
  if (p.b.D <= 32 && p.b.O <= 32) launch<T, 32, 32, ACT, HP>(p, stream);
  else if (p.b.D <= 32) launch<T, 32, 64, ACT, HP>(p, stream);
  else if (p.b.O <= 32) launch<T, 64, 32, ACT, HP>(p, stream);
  else launch<T, 64, 64, ACT, HP>(p, stream);
}

template <class T, int HP>
void by_act(const NarrowArgs& p, hipStream_t stream) {
  if (p.b.act == FD_ACT_SILU) launch_narrow<T, FD_ACT_SILU, HP>(p, stream);
  else launch_narrow<T, FD_ACT_GELU, HP>(p, stream);
}

}  // namespace

void run_narrow(const NarrowArgs& p, int planes, hipStream_t stream) {
  if (p.b.type == FD_F32) by_act<float, 3>(p, stream);
  else if (planes == 2) by_act<bf16, 2>(p, stream);
  else by_act<bf16, 1>(p, stream);
}

}  // namespace net
}  // namespace fd
