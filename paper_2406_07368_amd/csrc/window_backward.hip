// Gradient of softmax attention over a sliding window with sinks, bf16 rows.  With P_ts = exp(scale q_t.k_s - lse_t),
//
//   dP = dO V^T,  dS = P (dP - delta),  delta_t = dout_t . out_t
//   dq = scale dS K,  dk = scale dS^T Q,  dv = P^T dO
//
// Two kernels, so that every gradient row has one owner and nothing is added atomically; each makes S and dP again (seven
// products of 2 d flops a visible pair where five would do).
//   rows of q    128 queries a workgroup, a wave's 32 in its lanes, keys 64 at a time through LDS, as in the prefill:
//                S^T = K Q^T, dP^T = V dO^T, and dS^T, packed, is the operand of dQ^T += K^T dS^T as it stands.  Writes
//                delta for the other kernel.
//   rows of k, v 128 keys of a key/value head a workgroup, a wave's 32 in its lanes, queries 64 at a time through LDS,
//                over all query heads that share the keys: S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS.
// Key tile 0 would meet every query of the sequence for the sake of its sinks, many times what other tiles have to do: the
// query tiles that see nothing of it but sinks are shared out over workgroups of their own, whose sums (fp32, per wave)
// go to the workspace and are added up in a fixed order by a third launch.
//
// Bound: the matrix cores (14 d flops a visible pair here).
#include "common.h"
#include "kernels.h"
#include "mfma_util.h"
#include "window.h"

namespace linattn {

namespace {

template <int D>
struct Cfg {
  static constexpr int RS = D + 16;
  static constexpr int BUF = 2 * 64 * RS;       // elements of one buffer: 64 rows of two tensors
  static constexpr int BYTES = 2 * BUF * 2 + 4 * 64 * 4;   // ... and (rows of k, v) lse and delta, two buffers
  static constexpr int OS = D + 8;
  static constexpr int PPR = D / 8;
  static constexpr int NP = 64 * PPR / 256;
  static constexpr int CT = D / 32, KS = D / 16;
  static_assert(128 * OS <= 2 * BUF, "the finished rows take the buffers' place");
};

// 128 finished rows, X^T in accumulators (a row per lane of each wave, its elements in the registers) -> whole rows
template <int D>
__device__ __forceinline__ void store_tile(uint16_t* smem, const f32x16 (&X)[D / 32], float f, uint16_t* out, int64_t st, int r0, int r_end, int len, int tid) {
  using G = Cfg<D>;
  const int w = tid >> 6, lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  __syncthreads();
#pragma unroll
  for (int ct = 0; ct < G::CT; ++ct)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const u32x2 y = {pack_bf16x2(X[ct][4 * r4] * f, X[ct][4 * r4 + 1] * f), pack_bf16x2(X[ct][4 * r4 + 2] * f, X[ct][4 * r4 + 3] * f)};
      *reinterpret_cast<u32x2*>(smem + (32 * w + l32) * G::OS + 32 * ct + 8 * r4 + 4 * hi) = y;
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 128 * G::PPR / 256; ++i) {
    const int p = tid + 256 * i, r = p / G::PPR;
    const u32x4 x = *reinterpret_cast<const u32x4*>(smem + r * G::OS + p % G::PPR * 8), z = {0u, 0u, 0u, 0u};
    if (r0 + r < r_end) *reinterpret_cast<u32x4*>(out + (r0 + r) * st + p % G::PPR * 8) = r0 + r < len ? x : z;
  }
}

template <int D>
__device__ __forceinline__ void zero_rows(uint16_t* out, int64_t st, int r0, int r_end, int tid) {
  constexpr int PPR = D / 8;
  for (int e = tid; e < (r_end - r0) * PPR; e += 256) *reinterpret_cast<u32x4*>(out + (r0 + e / PPR) * st + e % PPR * 8) = u32x4{0u, 0u, 0u, 0u};
}

template <int D>
__global__ __launch_bounds__(256, 2) void window_dq_kernel(WindowArgs a, int n) {
  using G = Cfg<D>;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  const int place = xcd_place(blockIdx.x, n);
  if (place >= n) return;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int group = a.H / a.Hkv, ntile = (a.L + 127) / 128;
  const int g = place % group, tile = place / group % ntile, bk = place / group / ntile;
  const int b = bk / a.Hkv, hk = bk % a.Hkv, h = hk * group + g;
  const int len = clamp_len(a.lens, b, a.L);
  const int t0 = tile * 128, t_end = t0 + 128 < a.L ? t0 + 128 : a.L;
  uint16_t* gdq = const_cast<uint16_t*>(static_cast<const uint16_t*>(a.dq.p)) + b * a.dq.b + h * a.dq.h;
  const int64_t stat = ((int64_t)b * a.H + h) * a.L;
  if (t0 >= len) {
    zero_rows<D>(gdq, a.dq.t, t0, t_end, tid);
    return;
  }
  const uint16_t* gk = static_cast<const uint16_t*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const uint16_t* gv = static_cast<const uint16_t*>(a.v.p) + b * a.v.b + hk * a.v.h;
  const float c = window_log2_scale(a.scale);
  const int t = t0 + 32 * w + l32, tw = t0 + 32 * w, tr = t < len ? t : len - 1;
  bf16x8 qop[G::KS], dop[G::KS];
  float delta = 0.f;
  {
    const uint16_t* pq = static_cast<const uint16_t*>(a.q.p) + b * a.q.b + h * a.q.h + tr * a.q.t + 8 * hi;
    const uint16_t* pd = static_cast<const uint16_t*>(a.dout.p) + b * a.dout.b + h * a.dout.h + tr * a.dout.t + 8 * hi;
    const uint16_t* po = static_cast<const uint16_t*>(a.out.p) + b * a.out.b + h * a.out.h + tr * a.out.t + 8 * hi;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) {
      qop[ks] = *reinterpret_cast<const bf16x8*>(pq + 16 * ks);
      dop[ks] = *reinterpret_cast<const bf16x8*>(pd + 16 * ks);
      const bf16x8 o = *reinterpret_cast<const bf16x8*>(po + 16 * ks);
#pragma unroll
      for (int j = 0; j < 8; ++j) delta += (float)dop[ks][j] * (float)o[j];
    }
  }
  delta = add_xor32(delta);
  if (hi == 0 && t < len) a.delta[stat + t] = delta;
  const float lse2 = a.lse[stat + tr] * 1.44269504088896340736f;

  const int last = (t_end < len ? t_end : len) - 1;
  const int lo = (t0 - a.window + 1 > 0 ? t0 - a.window + 1 : 0) / 64;
  const int ns = a.sinks > 0 && lo > 0 ? 1 : 0;
  const int nk = ns + last / 64 - lo + 1;
  auto key0 = [&](int i) { return (i < ns ? i : lo + i - ns) * 64; };
  u32x4 rk[G::NP], rv[G::NP];
  auto request = [&](int s0) {
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + 256 * i, s = s0 + p / G::PPR, e = p % G::PPR * 8;
      const int row = s < len ? s : 0;
      rk[i] = *reinterpret_cast<const u32x4*>(gk + row * a.k.t + e);
      rv[i] = *reinterpret_cast<const u32x4*>(gv + row * a.v.t + e);
    }
  };
  auto put = [&](int s0, uint16_t* buf) {
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + 256 * i;
      uint16_t* d = buf + p / G::PPR * G::RS + p % G::PPR * 8;
      const u32x4 z = {0u, 0u, 0u, 0u};
      const bool in = s0 + p / G::PPR < len;
      *reinterpret_cast<u32x4*>(d) = in ? rk[i] : z;
      *reinterpret_cast<u32x4*>(d + 64 * G::RS) = in ? rv[i] : z;
    }
  };
  f32x16 dQ[G::CT];
#pragma unroll
  for (int i = 0; i < G::CT; ++i) dQ[i] = f32x16{};
  request(key0(0));
  put(key0(0), smem);
  for (int i = 0; i < nk; ++i) {
    const int s0 = key0(i);
    const uint16_t *Kl = smem + (i & 1) * G::BUF, *Vl = Kl + 64 * G::RS;
    __syncthreads();
    if (i + 1 < nk) request(key0(i + 1));
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int sw = s0 + 32 * kt;
      if (!(sw <= tw + 31 && (sw + 31 > tw - a.window || sw < a.sinks))) continue;
      f32x16 x = {}, y = {};
#pragma unroll
      for (int ks = 0; ks < G::KS; ++ks) {
        x = mfma(lds_row8(Kl + (32 * kt + l32) * G::RS + 16 * ks + 8 * hi), qop[ks], x);
        y = mfma(lds_row8(Vl + (32 * kt + l32) * G::RS + 16 * ks + 8 * hi), dop[ks], y);
      }
      const bool all = sw + 31 <= tw && (sw > tw + 31 - a.window || sw + 32 <= a.sinks);
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(x[r] * c - lse2) * (y[r] - delta);
      if (!all) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!window_sees(t, sw + acc_row(r, hi), a.window, a.sinks)) x[r] = 0.f;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8 p = pack8(x, 8 * half);
#pragma unroll
        for (int ct = 0; ct < G::CT; ++ct) dQ[ct] = mfma(tr_operand_acc_order(Kl, G::RS, 32 * kt + 16 * half, 32 * ct, lane), p, dQ[ct]);
      }
    }
    if (i + 1 < nk) put(key0(i + 1), smem + ((i + 1) & 1) * G::BUF);
  }
  store_tile<D>(smem, dQ, a.scale, gdq, a.dq.t, t0, t_end, len, tid);
}

// SINKS: the query tiles beyond window_far_tile of key tile 0; the waves take (32 keys, 32 queries) each.
template <int D, bool SINKS>
__global__ __launch_bounds__(256, 1) void window_dkv_kernel(WindowArgs a, int n) {
  using G = Cfg<D>;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  float* stats = reinterpret_cast<float*>(smem + 2 * G::BUF);    // [2][lse | delta][64]
  const int place = SINKS ? (int)blockIdx.x : xcd_place(blockIdx.x, n);
  if (place >= n) return;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int group = a.H / a.Hkv, ntile = SINKS ? a.far : (a.L + 127) / 128;
  const int tile = place % ntile, bk = place / ntile;
  const int b = bk / a.Hkv, hk = bk % a.Hkv;
  const int len = clamp_len(a.lens, b, a.L);
  const int s0 = SINKS ? 0 : tile * 128, s_end = s0 + 128 < a.L ? s0 + 128 : a.L;
  uint16_t* gdk = const_cast<uint16_t*>(static_cast<const uint16_t*>(a.dk.p)) + b * a.dk.b + hk * a.dk.h;
  uint16_t* gdv = const_cast<uint16_t*>(static_cast<const uint16_t*>(a.dv.p)) + b * a.dv.b + hk * a.dv.h;
  if (!SINKS && s0 >= len && !(a.far > 0 && s0 == 0)) {
    zero_rows<D>(gdk, a.dk.t, s0, s_end, tid);
    zero_rows<D>(gdv, a.dv.t, s0, s_end, tid);
    return;
  }
  const float c = window_log2_scale(a.scale);
  const int kw = SINKS ? 32 * (w & 1) : s0 + 32 * w;             // the wave's first key
  const int s = kw + l32;                                        // this lane's key
  bf16x8 kop[G::KS], vop[G::KS];
  {
    const int row = s < len ? s : 0;
    const uint16_t* pk = static_cast<const uint16_t*>(a.k.p) + b * a.k.b + hk * a.k.h + row * a.k.t + 8 * hi;
    const uint16_t* pv = static_cast<const uint16_t*>(a.v.p) + b * a.v.b + hk * a.v.h + row * a.v.t + 8 * hi;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) {
      kop[ks] = *reinterpret_cast<const bf16x8*>(pk + 16 * ks);
      vop[ks] = *reinterpret_cast<const bf16x8*>(pv + 16 * ks);
    }
  }
  // query tiles of one head: q_lo .. q_hi - 1; this workgroup's items are (head of the group, tile)
  const int q_len = (len + 63) / 64;
  const int far0 = window_far_tile(a.window);
  int q_lo, q_n, first, step;
  if (SINKS) {
    q_lo = far0; q_n = q_len > far0 ? q_len - far0 : 0;
    first = tile; step = a.far;
  } else {
    q_lo = s0 / 64;
    const int64_t end = ((int64_t)s0 + 127 + a.window - 1) / 64 + 1;   // (key tile 0: window_far_tile)
    q_n = q_len < end ? q_len - q_lo : (int)end - q_lo;
    if (q_n < 0) q_n = 0;
    first = 0; step = 1;
  }
  const int items = q_n * group;

  u32x4 rq[G::NP], rd[G::NP];
  float rs = 0.f;
  auto request = [&](int it) {
    const int h = hk * group + it / q_n, t0 = (q_lo + it % q_n) * 64;
    const uint16_t* gq = static_cast<const uint16_t*>(a.q.p) + b * a.q.b + h * a.q.h;
    const uint16_t* gd = static_cast<const uint16_t*>(a.dout.p) + b * a.dout.b + h * a.dout.h;
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + 256 * i, t = t0 + p / G::PPR, e = p % G::PPR * 8;
      const int row = t < len ? t : 0;
      rq[i] = *reinterpret_cast<const u32x4*>(gq + row * a.q.t + e);
      rd[i] = *reinterpret_cast<const u32x4*>(gd + row * a.dout.t + e);
    }
    if (tid < 128) {
      const int t = t0 + (tid & 63);
      const int64_t at = ((int64_t)b * a.H + h) * a.L + t;
      rs = t < len ? (tid < 64 ? a.lse[at] * 1.44269504088896340736f : a.delta[at]) : 0.f;
    }
  };
  auto put = [&](int it, int which) {
    const int t0 = (q_lo + it % q_n) * 64;
    uint16_t* buf = smem + which * G::BUF;
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + 256 * i;
      uint16_t* d = buf + p / G::PPR * G::RS + p % G::PPR * 8;
      const u32x4 z = {0u, 0u, 0u, 0u};
      const bool in = t0 + p / G::PPR < len;
      *reinterpret_cast<u32x4*>(d) = in ? rq[i] : z;
      *reinterpret_cast<u32x4*>(d + 64 * G::RS) = in ? rd[i] : z;
    }
    if (tid < 128) stats[which * 128 + tid] = rs;
  };

  f32x16 dK[G::CT], dV[G::CT];
#pragma unroll
  for (int i = 0; i < G::CT; ++i) { dK[i] = f32x16{}; dV[i] = f32x16{}; }
  if (first < items) {
    request(first);
    put(first, 0);
  }
  for (int it = first, par = 0; it < items; it += step, par ^= 1) {
    const int t0 = (q_lo + it % q_n) * 64;
    const uint16_t *Ql = smem + par * G::BUF, *dl = Ql + 64 * G::RS;
    const float* st = stats + par * 128;
    __syncthreads();
    if (it + step < items) request(it + step);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int tw = t0 + 32 * tt;
      if (SINKS ? (tt != w >> 1 || kw >= a.sinks || tw >= len) : !(kw <= tw + 31 && (kw + 31 > tw - a.window || kw < a.sinks) && tw < len)) continue;
      f32x16 x = {}, y = {};
#pragma unroll
      for (int ks = 0; ks < G::KS; ++ks) {
        x = mfma(lds_row8(Ql + (32 * tt + l32) * G::RS + 16 * ks + 8 * hi), kop[ks], x);
        y = mfma(lds_row8(dl + (32 * tt + l32) * G::RS + 16 * ks + 8 * hi), vop[ks], y);
      }
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 le = *reinterpret_cast<const f32x4*>(st + 32 * tt + 8 * r4 + 4 * hi);
        const f32x4 de = *reinterpret_cast<const f32x4*>(st + 64 + 32 * tt + 8 * r4 + 4 * hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[4 * r4 + i] = __builtin_amdgcn_exp2f(x[4 * r4 + i] * c - le[i]);
          y[4 * r4 + i] = x[4 * r4 + i] * (y[4 * r4 + i] - de[i]);
        }
      }
      const bool all = kw + 31 <= tw && (kw > tw + 31 - a.window || kw + 32 <= a.sinks) && tw + 32 <= len;
      if (!all) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int t = tw + acc_row(r, hi);
          if (!(window_sees(t, s, a.window, a.sinks) && t < len)) { x[r] = 0.f; y[r] = 0.f; }
        }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8 p = pack8(x, 8 * half), ds = pack8(y, 8 * half);
#pragma unroll
        for (int ct = 0; ct < G::CT; ++ct) {
          dV[ct] = mfma(tr_operand_acc_order(dl, G::RS, 32 * tt + 16 * half, 32 * ct, lane), p, dV[ct]);
          dK[ct] = mfma(tr_operand_acc_order(Ql, G::RS, 32 * tt + 16 * half, 32 * ct, lane), ds, dK[ct]);
        }
      }
    }
    if (it + step < items) put(it + step, par ^ 1);
  }
  if (!SINKS) {
    store_tile<D>(smem, dK, a.scale, gdk, a.dk.t, s0, s_end, len, tid);
    store_tile<D>(smem, dV, 1.f, gdv, a.dv.t, s0, s_end, len, tid);
  }
  // the sinks' shares: slot 0 what key tile 0 met in its own query tiles, then a slot for each wave half of each SINKS workgroup
  if (a.far > 0 && s0 == 0 && s < a.sinks) {
    const int slot = SINKS ? 1 + 2 * tile + (w >> 1) : 0;
    float* p = a.part + (((int64_t)bk * (1 + 2 * a.far) + slot) * 2 * a.sinks + s) * D;
#pragma unroll
    for (int ct = 0; ct < G::CT; ++ct)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int e = 32 * ct + 8 * r4 + 4 * hi;
        *reinterpret_cast<f32x4*>(p + e) = f32x4{dK[ct][4 * r4], dK[ct][4 * r4 + 1], dK[ct][4 * r4 + 2], dK[ct][4 * r4 + 3]};
        *reinterpret_cast<f32x4*>(p + (int64_t)a.sinks * D + e) = f32x4{dV[ct][4 * r4], dV[ct][4 * r4 + 1], dV[ct][4 * r4 + 2], dV[ct][4 * r4 + 3]};
      }
  }
}

// a sink row's gradient: the sum of its shares, a wave per row of dk or dv
template <int D>
__global__ __launch_bounds__(64) void window_sinks_kernel(WindowArgs a) {
  const int s = blockIdx.x % a.sinks, kv = blockIdx.x / a.sinks % 2, bk = blockIdx.x / (2 * a.sinks);
  const int b = bk / a.Hkv, hk = bk % a.Hkv, slots = 1 + 2 * a.far;
  const Rows& o = kv ? a.dv : a.dk;
  uint16_t* out = const_cast<uint16_t*>(static_cast<const uint16_t*>(o.p)) + b * o.b + hk * o.h + s * o.t;
  const bool in = s < clamp_len(a.lens, b, a.L);
  for (int e = threadIdx.x; e < D; e += 64) {
    const float* p = a.part + (((int64_t)bk * slots * 2 + kv) * a.sinks + s) * D + e;
    float x = 0.f;
    for (int i = 0; i < slots; ++i) x += p[(int64_t)i * 2 * a.sinks * D];
    out[e] = in ? f32_to_bf16_bits(kv ? x : x * a.scale) : 0;
  }
}

template <int D>
hipError_t launch(const WindowArgs& a, hipStream_t s) {
  const int nq = a.B * a.H * ((a.L + 127) / 128), nk = a.B * a.Hkv * ((a.L + 127) / 128);
  hipError_t e = LINATTN_MAX_LDS_ONCE((window_dq_kernel<D>), Cfg<D>::BYTES);
  if (e != hipSuccess) return e;
  e = LINATTN_MAX_LDS_ONCE((window_dkv_kernel<D, false>), Cfg<D>::BYTES);
  if (e != hipSuccess) return e;
  window_dq_kernel<D><<<dim3((nq + 7) / 8 * 8), 256, Cfg<D>::BYTES, s>>>(a, nq);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.far > 0) {
    e = LINATTN_MAX_LDS_ONCE((window_dkv_kernel<D, true>), Cfg<D>::BYTES);
    if (e != hipSuccess) return e;
    window_dkv_kernel<D, true><<<dim3(a.B * a.Hkv * a.far), 256, Cfg<D>::BYTES, s>>>(a, a.B * a.Hkv * a.far);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  window_dkv_kernel<D, false><<<dim3((nk + 7) / 8 * 8), 256, Cfg<D>::BYTES, s>>>(a, nk);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.far > 0) {
    window_sinks_kernel<D><<<dim3(a.B * a.Hkv * 2 * a.sinks), 64, 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_window_backward(const WindowArgs& a, int d, hipStream_t s) { return d == 64 ? launch<64>(a, s) : launch<128>(a, s); }

}  // namespace linattn
