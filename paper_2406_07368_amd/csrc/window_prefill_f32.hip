// Softmax attention over a sliding window with sinks, fp32 rows, in exact fp32 products (v_mfma_f32_32x32x2_f32).  The
// scheme is window_prefill.hip's with 32 keys at a time: 128 or 64 queries a workgroup, 32 a wave, a query per lane, one pass
// with a running maximum and sum.  A register of the score accumulator holds the keys s (low half of the wave) and s + 4
// (high half), which is an operand of the fp32 instruction as it stands: the weights move nowhere.  The two halves of a
// wave contract the two halves of the features.
//
// Bound: the fp32 matrix rate (4 d flops a visible pair): 97 TFLOP/s at 64 heads of 4096 tokens, d = 128, a window of 1024.
#include "common.h"
#include "kernels.h"
#include "window.h"

namespace linattn {

namespace {

constexpr int KT = 32;

template <int D, int QT>
struct Cfg {
  static constexpr int NT = 2 * QT;              // a wave for 32 queries
  static constexpr int RS = D + 4;
  static constexpr int PPR = D / 4;
  static constexpr int NP = KT * PPR / NT;
  static constexpr int FLOATS = QT * RS > 2 * KT * RS ? QT * RS : 2 * KT * RS;   // finished rows; K, V
};

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

template <int D, int QT>
__global__ __launch_bounds__(2 * QT, 2) void window_prefill_f32_kernel(WindowArgs a) {
  using G = Cfg<D, QT>;
  extern __shared__ __attribute__((aligned(16))) float smem_f[];
  const int group = a.H / a.Hkv, ntile = (a.L + QT - 1) / QT;
  const int place = xcd_place(blockIdx.x, a.B * a.Hkv, group * ntile);
  const int g = place % group, tile = place / group % ntile, bk = place / group / ntile;
  if (bk >= a.B * a.Hkv) return;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int b = bk / a.Hkv, hk = bk % a.Hkv, h = hk * group + g;
  const int len = clamp_len(a.lens, b, a.L);
  const int t0 = tile * QT, t_end = t0 + QT < a.L ? t0 + QT : a.L;
  float* gout = const_cast<float*>(static_cast<const float*>(a.out.p)) + b * a.out.b + h * a.out.h;
  float* glse = a.lse ? a.lse + ((int64_t)b * a.H + h) * a.L : nullptr;
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};
  if (t0 >= len) {
    for (int e = tid; e < (t_end - t0) * G::PPR; e += G::NT) *reinterpret_cast<f32x4*>(gout + (t0 + e / G::PPR) * a.out.t + e % G::PPR * 4) = z;
    if (glse)
      for (int t = t0 + tid; t < t_end; t += G::NT) glse[t] = -__builtin_inff();
    return;
  }
  const float* gq = static_cast<const float*>(a.q.p) + b * a.q.b + h * a.q.h;
  const float* gk = static_cast<const float*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const float* gv = static_cast<const float*>(a.v.p) + b * a.v.b + hk * a.v.h;
  const float c = window_log2_scale(a.scale);
  float *Kl = smem_f, *Vl = smem_f + KT * G::RS;

  const int t = t0 + 32 * w + l32, tw = t0 + 32 * w;
  f32x4 qop[D / 8];
  {
    const float* p = gq + (t < len ? t : len - 1) * a.q.t + D / 2 * hi;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) qop[i] = *reinterpret_cast<const f32x4*>(p + 4 * i);
  }
  const int last = (t_end < len ? t_end : len) - 1;
  const int lo = (t0 - a.window + 1 > 0 ? t0 - a.window + 1 : 0) / KT;
  const int sink_tiles = (a.sinks + KT - 1) / KT, ns = sink_tiles < lo ? sink_tiles : lo;
  const int nk = ns + last / KT - lo + 1;
  auto key0 = [&](int i) { return (i < ns ? i : lo + i - ns) * KT; };

  f32x4 rk[G::NP], rv[G::NP];
  auto request = [&](int s0) {
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + G::NT * i, s = s0 + p / G::PPR, e = p % G::PPR * 4;
      const int row = s < len ? s : 0;
      rk[i] = *reinterpret_cast<const f32x4*>(gk + row * a.k.t + e);
      rv[i] = *reinterpret_cast<const f32x4*>(gv + row * a.v.t + e);
    }
  };
  f32x16 O[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) O[i] = f32x16{};
  float m = -__builtin_inff(), l = 0.f;

  request(key0(0));
  for (int i = 0; i < nk; ++i) {
    const int s0 = key0(i);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < G::NP; ++j) {
      const int p = tid + G::NT * j;
      float* d = Kl + p / G::PPR * G::RS + p % G::PPR * 4;
      const bool in = s0 + p / G::PPR < len;
      *reinterpret_cast<f32x4*>(d) = in ? rk[j] : z;
      *reinterpret_cast<f32x4*>(d + KT * G::RS) = in ? rv[j] : z;
    }
    __syncthreads();
    if (i + 1 < nk) request(key0(i + 1));
    if (!(s0 <= tw + 31 && (s0 + KT - 1 > tw - a.window || s0 < a.sinks))) continue;
    f32x16 x = {};
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      const f32x4 kk = *reinterpret_cast<const f32x4*>(Kl + l32 * G::RS + D / 2 * hi + 4 * j);
#pragma unroll
      for (int e = 0; e < 4; ++e) x = mfma_f32(kk[e], qop[j][e], x);
    }
    const bool all = s0 + KT - 1 <= tw && (s0 > tw + 31 - a.window || s0 + KT <= a.sinks);
    if (!all) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!window_sees(t, s0 + acc_row(r, hi), a.window, a.sinks)) x[r] = -__builtin_inff();
    }
    float top = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, x[r]);
    const float m2 = fmaxf(m, max_xor32(top) * c);
    const float mm = m2 == -__builtin_inff() ? 0.f : m2;
    const float f = __builtin_amdgcn_exp2f(m - mm);
    m = m2;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r] = __builtin_amdgcn_exp2f(x[r] * c - mm);
      sum += x[r];
    }
    l = l * f + sum;
    if (__any(f != 1.f)) {
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct) O[ct] *= f;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct) O[ct] = mfma_f32(Vl[acc_row(r, hi) * G::RS + 32 * ct + l32], x[r], O[ct]);
  }

  l = add_xor32(l);
  const bool in = t < len;
  const float inv = in ? 1.f / l : 0.f;
  if (glse && hi == 0 && t < t_end) glse[t] = in ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : -__builtin_inff();
  __syncthreads();
#pragma unroll
  for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const f32x4 y = {O[ct][4 * r4] * inv, O[ct][4 * r4 + 1] * inv, O[ct][4 * r4 + 2] * inv, O[ct][4 * r4 + 3] * inv};
      *reinterpret_cast<f32x4*>(smem_f + (32 * w + l32) * G::RS + 32 * ct + 8 * r4 + 4 * hi) = y;
    }
  __syncthreads();
#pragma unroll 4
  for (int i = 0; i < QT * G::PPR / G::NT; ++i) {
    const int p = tid + G::NT * i, r = p / G::PPR;
    const f32x4 x = *reinterpret_cast<const f32x4*>(smem_f + r * G::RS + p % G::PPR * 4);
    if (t0 + r < t_end) *reinterpret_cast<f32x4*>(gout + (t0 + r) * a.out.t + p % G::PPR * 4) = t0 + r < len ? x : z;
  }
}

template <int D, int QT>
hipError_t launch(const WindowArgs& a, hipStream_t s) {
  using G = Cfg<D, QT>;
  hipError_t e = LINATTN_MAX_LDS_ONCE((window_prefill_f32_kernel<D, QT>), G::FLOATS * 4);
  if (e != hipSuccess) return e;
  window_prefill_f32_kernel<D, QT><<<dim3((unsigned)xcd_grid(a.B * a.Hkv, a.H / a.Hkv * ((a.L + QT - 1) / QT))), G::NT, G::FLOATS * 4, s>>>(a);
  return hipGetLastError();
}
}  // namespace

// Rows of 64 in fewer than 512 workgroups of 128 queries (two a compute unit): of 64 queries instead, which spread more
// evenly: 66 -> 58 us at 48 heads of 1001 tokens, the same from there on.  (Rows of 128: 82 -> 121 us at 32 heads of 1024.)
hipError_t launch_window_prefill_f32(const WindowArgs& a, int d, hipStream_t s) {
  if (d == 128) return launch<128, 128>(a, s);
  return (int64_t)a.B * a.H * ((a.L + 127) / 128) < 512 ? launch<64, 64>(a, s) : launch<64, 128>(a, s);
}

}  // namespace linattn
