// Gradient of softmax attention over a sliding window with sinks, bf16 rows.  With P_ts = exp(scale q_t.k_s - lse_t),
//
//   dP = dO V^T,  dS = P (dP - delta),  delta_t = dout_t . out_t
//   dq = scale dS K,  dk = scale dS^T Q,  dv = P^T dO
//
// Two kernels, so that every gradient row has one owner and nothing is added atomically; each makes S and dP again (seven
// products of 2 d flops a visible pair where five would do).
//   rows of q    128 queries a workgroup, a wave's 32 in its lanes, keys 64 at a time through LDS, as in the prefill:
//                S^T = K Q^T, dP^T = V dO^T, and dS^T, packed, is the operand of dQ^T += K^T dS^T as it stands.  Writes
//                lse (in base 2) and delta for the other kernel.
//   rows of k, v 128 keys of a key/value head a workgroup, a wave's 32 in its lanes, queries 32 at a time through LDS,
//                over all query heads that share the keys: S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS.  The
//                value rows stay in LDS and not in registers, so that two waves fit a SIMD.
// Key tile 0 would meet every query of the sequence for the sake of its sinks, many times what other tiles have to do: the
// query tiles that see nothing of it but sinks are shared out over workgroups of their own, and where there are few key
// tiles each is shared by several workgroups.  Their sums (fp32) go to the workspace and are added up in a fixed order.
//
// P and dS are rounded to bf16 once for the products, whose sums are fp32: the gradients are off by 2.35e-3 in the 2-norm, of which their
// own rounding is 1.66e-3.  In two terms each 1.67e-3, for dq 185 -> 225 us, dk and dv 300 -> 411.
//
// Bound (14 d flops a visible pair here): no unit alone.  dq: matrix cores 48 % of the cycles, vector ALUs 35, LDS 26; dk and dv: 38, 28 and
// 29 -- two waves on a SIMD, whose accumulators leave registers for operands one step ahead, wait for each other's units in turn.
// Measured at 64 heads of 128 over sequences of up to 4096 tokens, a window of 1024: dq 183 us, 840 TFLOP/s; dk and dv 300 to 321 us
// (boards differ), 650 TFLOP/s.
#include "common.h"
#include "kernels.h"
#include "mfma_util.h"
#include "window.h"

namespace linattn {

namespace {

template <int D>
struct Cfg {
  static constexpr int BUF = 2 * 64 * D;        // elements of one buffer: 64 rows of two tensors
  static constexpr int OS = D + 8;
  static constexpr int TILES = (2 * BUF > 128 * OS ? 2 * BUF : 128 * OS) * 2;   // bytes: the buffers; finished rows
  static constexpr int DKV = (128 + 4 * kWindowQ) * D * 2 > 128 * OS * 2 ? (128 + 4 * kWindowQ) * D * 2 : 128 * OS * 2;   // value rows, two buffers; finished rows
  static constexpr int DKV_BYTES = DKV + 4 * kWindowQ * 4;   // ... and lse and delta, two buffers
  static constexpr int PPR = D / 8;
  static constexpr int CT = D / 32, KS = D / 16;
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
__global__ __launch_bounds__(256, 2) void window_dq_kernel(WindowArgs a) {
  using G = Cfg<D>;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  const int group = a.H / a.Hkv, ntile = (a.L + 127) / 128;
  const int place = xcd_place(blockIdx.x, a.B * a.Hkv, group * ntile);
  const int g = place % group, tile = place / group % ntile, bk = place / group / ntile;
  if (bk >= a.B * a.Hkv) return;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
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
  const Swizzled<D> lds(lane, 4);
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
  const float lse2 = a.lse[stat + tr] * 1.44269504088896340736f;

  const int last = (t_end < len ? t_end : len) - 1;
  const int lo = (t0 - a.window + 1 > 0 ? t0 - a.window + 1 : 0) / 64;
  const int ns = a.sinks > 0 && lo > 0 ? 1 : 0;
  const int nk = ns + last / 64 - lo + 1;
  auto key0 = [&](int i) { return (i < ns ? i : lo + i - ns) * 64; };
  const Fetch<D> fetch(tid);
  auto request = [&](int i, uint16_t* buf) {
    const int s0 = key0(i);
    fetch.request(buf, gk + s0 * a.k.t, a.k.t, len - s0);
    fetch.request(buf + 64 * D, gv + s0 * a.v.t, a.v.t, len - s0);
  };
  auto arrive = [&](int i, uint16_t* buf) {
    const int n = len - key0(i);
    fetch.arrived();
    fetch.trim(buf, n, tid);
    fetch.trim(buf + 64 * D, n, tid);
    __syncthreads();
  };
  constexpr int AHEAD = 3;
  auto visible = [&](int sw) { return sw <= tw + 31 && (sw + 31 > tw - a.window || sw < a.sinks); };
  uint16_t *even = smem, *odd = smem + G::BUF;
  // A row that sees n keys has an out of 1 / sqrt(n) of a value row, and so much of out's rounding to bf16 is in delta: where n is
  // small the gradient would be off by more than all of its own roundings.  There delta is summed up from the weights, in a pass of
  // its own over at most four key tiles (16 -> 18 us where a sequence has no other; nothing at the size above).
  if (t0 == 0 || (int64_t)a.window + a.sinks < 64) {
    float sum = 0.f;
    auto turn = [&](int i, uint16_t* cur, uint16_t* next) {
      arrive(i, cur);
      if (i + 1 < nk) request(i + 1, next);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int sw = key0(i) + 32 * kt;
        if (!visible(sw)) continue;
        f32x16 x = {}, y = {};
#pragma unroll
        for (int ks = 0; ks < G::KS; ++ks) {
          x = mfma(lds.rows(cur, 32 * kt, ks), qop[ks], x);
          y = mfma(lds.rows(cur + 64 * D, 32 * kt, ks), dop[ks], y);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (window_sees(t, sw + acc_row(r, hi), a.window, a.sinks)) sum += __builtin_amdgcn_exp2f(x[r] * c - lse2) * y[r];
      }
    };
    request(0, even);
    for (int i = 0; i < nk; ++i) turn(i, i % 2 ? odd : even, i % 2 ? even : odd);
    __syncthreads();
    delta = add_xor32(sum);
  }
  if (t < len) a.stats[hi * (int64_t)a.B * a.H * a.L + stat + t] = hi ? delta : lse2;

  // The weight of a token that sees only itself is 1 whatever the score: no gradient, which dP - delta would give only up to its
  // rounding.  (-1 sees nothing.  A tile with such a token is never one in which all is seen.)
  const int tm = t == 0 || (a.window == 1 && a.sinks == 0) ? -1 : t;
  f32x16 dQ[G::CT];
#pragma unroll
  for (int i = 0; i < G::CT; ++i) dQ[i] = f32x16{};
  auto tile_of = [&](int i, const uint16_t* Kl) {
    const uint16_t* Vl = Kl + 64 * D;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int sw = key0(i) + 32 * kt;
      if (!visible(sw)) continue;
      // the matrix operands in the order of their use, AHEAD of each kind read before they are needed
      bf16x8 ko[G::KS], vo[G::KS], kt_op[2 * G::CT];
      auto read = [&](int j) {
        if (j < G::KS) {
          ko[j] = lds.rows(Kl, 32 * kt, j);
          vo[j] = lds.rows(Vl, 32 * kt, j);
        } else if (j < G::KS + 2 * G::CT) {
          const int n = j - G::KS;
          kt_op[n] = lds.cols_acc(Kl, 32 * kt + 16 * (n / G::CT), n % G::CT);
        }
      };
      f32x16 x = {}, y = {};
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) read(j);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < G::KS; ++ks) {
        x = mfma(ko[ks], qop[ks], x);
        y = mfma(vo[ks], dop[ks], y);
        read(ks + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
      const bool all = sw + 31 <= tw && (sw > tw + 31 - a.window || sw + 32 <= a.sinks);
      auto weigh = [&](int from, int to) {
#pragma unroll
        for (int r = from; r < to; ++r) x[r] = __builtin_amdgcn_exp2f(x[r] * c - lse2) * (y[r] - delta);
      };
      weigh(0, 8);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (!all) {
#pragma unroll
          for (int r = 8 * half; r < 8 * half + 8; ++r)
            if (!window_sees(tm, sw + acc_row(r, hi), a.window, a.sinks)) x[r] = 0.f;
        }
        const bf16x8 p = pack8(x, 8 * half);
#pragma unroll
        for (int ct = 0; ct < G::CT; ++ct) {
          __builtin_amdgcn_sched_barrier(0);
          dQ[ct] = mfma(kt_op[G::CT * half + ct], p, dQ[ct]);
          read(G::KS + G::CT * half + ct + AHEAD);
          if (half == 0) weigh(8 + 8 * ct / G::CT, 8 + 8 * (ct + 1) / G::CT);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  auto turn = [&](int i, uint16_t* __restrict cur, uint16_t* __restrict next) {   // (see Fetch)
    arrive(i, cur);
    if (i + 1 < nk) request(i + 1, next);
    tile_of(i, cur);
  };
  request(0, even);
  for (int i = 0; i < nk; i += 2) {
    turn(i, even, odd);
    if (i + 1 < nk) turn(i + 1, odd, even);
  }
  store_tile<D>(smem, dQ, a.scale, gdq, a.dq.t, t0, t_end, len, tid);
}

// Jobs of a key/value head: `far` for the sinks (the query tiles from window_far_tile on, with the sinks of key tile 0; the
// waves take 32 keys each, and every other of its query tiles), then `parts` for every key tile.
template <int D>
__global__ __launch_bounds__(256, 2) void window_dkv_kernel(WindowArgs a) {
  using G = Cfg<D>;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  uint16_t* Vl = smem;                                           // the value rows of the keys
  float* stats = reinterpret_cast<float*>(smem + G::DKV / 2);    // [2][lse | delta][32]
  const int group = a.H / a.Hkv, each = a.far + a.parts * ((a.L + 127) / 128);
  const int place = xcd_place(blockIdx.x, a.B * a.Hkv, each);
  const int bk = place / each;
  if (bk >= a.B * a.Hkv) return;
  const bool sink_job = place % each < a.far;
  const int tile = sink_job ? 0 : (place % each - a.far) / a.parts;
  const int part = sink_job ? place % each : (place % each - a.far) % a.parts;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int b = bk / a.Hkv, hk = bk % a.Hkv;
  const int len = clamp_len(a.lens, b, a.L);
  const int s0 = tile * 128, s_end = s0 + 128 < a.L ? s0 + 128 : a.L;
  uint16_t* gdk = const_cast<uint16_t*>(static_cast<const uint16_t*>(a.dk.p)) + b * a.dk.b + hk * a.dk.h;
  uint16_t* gdv = const_cast<uint16_t*>(static_cast<const uint16_t*>(a.dv.p)) + b * a.dv.b + hk * a.dv.h;
  const bool shares = a.far > 0 && s0 == 0;                      // the sinks' rows are added up from shares
  if (s0 >= len && !shares) {
    if (part == 0) {
      zero_rows<D>(gdk, a.dk.t, s0, s_end, tid);
      zero_rows<D>(gdv, a.dv.t, s0, s_end, tid);
    }
    return;
  }
  const float c = window_log2_scale(a.scale);
  const Swizzled<D> lds(lane, 4);
  const int kw = sink_job ? 32 * (w & 1) : s0 + 32 * w;          // the wave's first key
  const int s = kw + l32;                                        // this lane's key
  bf16x8 kop[G::KS];
  {
    const int row = s < len ? s : 0;
    const uint16_t* pk = static_cast<const uint16_t*>(a.k.p) + b * a.k.b + hk * a.k.h + row * a.k.t + 8 * hi;
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) kop[ks] = *reinterpret_cast<const bf16x8*>(pk + 16 * ks);
  }
  const uint16_t* gv = static_cast<const uint16_t*>(a.v.p) + b * a.v.b + hk * a.v.h;
  const Fetch<D> vfetch(tid);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = s0 + 64 * i, n = len - r > 0 ? len - r : 0;    // (none: row 0 of the sequence, overwritten with zeros)
    vfetch.request(Vl + i * 64 * D, gv + (n > 0 ? r : 0) * a.v.t, a.v.t, n);
  }
  // query tiles of one head: q_lo .. q_lo + q_n - 1; the items are (head of the group, tile), every step-th of them this workgroup's
  const int q_len = (len + kWindowQ - 1) / kWindowQ;
  const int64_t near_end = ((int64_t)s0 + 127 + a.window - 1) / kWindowQ + 1;   // (key tile 0: window_far_tile)
  const int end = q_len < near_end ? q_len : (int)near_end;
  const int q_lo = sink_job ? end : s0 / kWindowQ;
  const int q_n = (sink_job ? q_len : end) - q_lo > 0 ? (sink_job ? q_len : end) - q_lo : 0;
  const int step = sink_job ? a.far : a.parts;
  // an item, in base q_n as it were, and the one a step on
  struct Item { int head, tile; };
  const int step_head = q_n > 0 ? step / q_n : 0, step_tile = q_n > 0 ? step % q_n : 0;
  auto after = [&](Item it) {
    it.head += step_head;
    it.tile += step_tile;
    if (it.tile >= q_n) { it.tile -= q_n; ++it.head; }
    return it;
  };

  const Fetch<D, kWindowQ> fetch(tid);
  auto first_row = [&](Item it) { return (q_lo + it.tile) * kWindowQ; };
  auto request = [&](Item it, uint16_t* buf, float* st) {
    const int h = hk * group + it.head, t0 = first_row(it), n = len - t0;
    fetch.request(buf, static_cast<const uint16_t*>(a.q.p) + b * a.q.b + h * a.q.h + t0 * a.q.t, a.q.t, n);
    fetch.request(buf + kWindowQ * D, static_cast<const uint16_t*>(a.dout.p) + b * a.dout.b + h * a.dout.h + t0 * a.dout.t, a.dout.t, n);
    if (w == 0) {                                // lanes: lse in base 2, then delta (behind the end: the last token's)
      const int r = lane % kWindowQ < n ? lane % kWindowQ : n - 1;
      const float* from = a.stats + (lane < kWindowQ ? 0 : (int64_t)a.B * a.H * a.L) + ((int64_t)b * a.H + h) * a.L + t0 + r;
      __builtin_amdgcn_global_load_lds((typename Fetch<D>::global_ptr)from, (typename Fetch<D>::lds_ptr)st, 4, 0, 0);
    }
  };
  auto arrive = [&](Item it, uint16_t* buf) {
    const int n = len - first_row(it);
    fetch.arrived();
    fetch.trim(buf, n, tid);
    fetch.trim(buf + kWindowQ * D, n, tid);
    __syncthreads();
  };

  f32x16 dK[G::CT], dV[G::CT];
#pragma unroll
  for (int i = 0; i < G::CT; ++i) { dK[i] = f32x16{}; dV[i] = f32x16{}; }
  auto tile_of = [&](Item it, int turn, const uint16_t* Ql, const float* st) {
    const uint16_t* dl = Ql + kWindowQ * D;
    const int tw = first_row(it);
    if (sink_job ? (turn & 1) != w >> 1 || kw >= a.sinks : !(kw <= tw + 31 && (kw + 31 > tw - a.window || kw < a.sinks))) return;
    int vo = (kw - s0) * D;
    Swizzled<D> at = lds;                        // (addresses kept over the loop would not fit the registers)
    asm volatile("" : "+s"(vo));
    at.forget_rows(); at.forget_cols();
    // the matrix operands in the order of their use, AHEAD of each kind read before they are needed (two: spills, which wait for the rows
    // under way, 613 -> 650 us)
    bf16x8 qo[G::KS], od[G::KS], vv[G::KS], dt[2 * G::CT], qt[2 * G::CT];
    auto read = [&](int i) {
      if (i < G::KS) {
        qo[i] = at.rows(Ql, 0, i);
        od[i] = at.rows(dl, 0, i);
        vv[i] = at.rows(Vl + vo, 0, i);
      } else if (i < G::KS + 2 * G::CT) {
        const int j = i - G::KS;
        dt[j] = at.cols_acc(dl, 16 * (j / G::CT), j % G::CT);
        qt[j] = at.cols_acc(Ql, 16 * (j / G::CT), j % G::CT);
      }
    };
    constexpr int AHEAD = 1;
    f32x16 x = {}, y = {};
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks) {
      x = mfma(qo[ks], kop[ks], x);
      y = mfma(od[ks], vv[ks], y);
      read(ks + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
    }
    const bool all = kw + 31 <= tw && (kw > tw + 31 - a.window || kw + 32 <= a.sinks) && tw + 32 <= len;
    auto weigh = [&](int r4) {
      const f32x4 le = *reinterpret_cast<const f32x4*>(st + 8 * r4 + 4 * hi);
      const f32x4 de = *reinterpret_cast<const f32x4*>(st + kWindowQ + 8 * r4 + 4 * hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[4 * r4 + i] = __builtin_amdgcn_exp2f(x[4 * r4 + i] * c - le[i]);
        y[4 * r4 + i] = x[4 * r4 + i] * (y[4 * r4 + i] - de[i]);
      }
    };
    auto mask = [&](int half) {
      if (!all) {
#pragma unroll
        for (int r = 8 * half; r < 8 * half + 8; ++r) {
          const int t = tw + acc_row(r, hi);
          if (!(window_sees(t, s, a.window, a.sinks) && t < len)) { x[r] = 0.f; y[r] = 0.f; }
        }
        if (half == 0 && tw == 0 && hi == 0) y[0] = 0.f;   // (acc_row(0, 0) is 0: token 0 sees only itself, as in dq)
      }
    };
    weigh(0); weigh(1);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      mask(half);
      const bf16x8 p = pack8(x, 8 * half), ds = pack8(y, 8 * half);
#pragma unroll
      for (int ct = 0; ct < G::CT; ++ct) {
        __builtin_amdgcn_sched_barrier(0);
        dV[ct] = mfma(dt[G::CT * half + ct], p, dV[ct]);
        dK[ct] = mfma(qt[G::CT * half + ct], ds, dK[ct]);
        read(G::KS + G::CT * half + ct + AHEAD);
        if (half == 0 && ct < 2) weigh(2 + ct);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  uint16_t *even = smem + 128 * D, *odd = even + 2 * kWindowQ * D;
  Item it = q_n > 0 ? Item{part / q_n, part % q_n} : Item{group, 0};
  if (it.head < group) request(it, even, stats);
  vfetch.arrived();
#pragma unroll
  for (int i = 0; i < 2; ++i) vfetch.trim(Vl + i * 64 * D, len - s0 - 64 * i, tid);
  auto one = [&](Item it, Item next_it, int turn, uint16_t* __restrict cur, float* __restrict st, uint16_t* __restrict next, float* __restrict st_next) {
    arrive(it, cur);
    if (next_it.head < group) request(next_it, next, st_next);
    tile_of(it, turn, cur, st);
  };
  for (int turn = 0; it.head < group; turn += 2) {
    const Item second = after(it);
    one(it, second, turn, even, stats, odd, stats + 2 * kWindowQ);
    it = after(second);
    if (second.head < group) one(second, it, turn + 1, odd, stats + 2 * kWindowQ, even, stats);
  }
  if (!sink_job && a.parts == 1) {
    store_tile<D>(smem, dK, a.dk_scale, gdk, a.dk.t, s0, s_end, len, tid);
    store_tile<D>(smem, dV, 1.f, gdv, a.dv.t, s0, s_end, len, tid);
  }
  // where the sums of this lane's key go, if they are a share: [2][rows][D], dk then dv
  auto give = [&](float* p, int64_t rows) {
#pragma unroll
    for (int ct = 0; ct < G::CT; ++ct)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int e = 32 * ct + 8 * r4 + 4 * hi;
        *reinterpret_cast<f32x4*>(p + e) = f32x4{dK[ct][4 * r4], dK[ct][4 * r4 + 1], dK[ct][4 * r4 + 2], dK[ct][4 * r4 + 3]};
        *reinterpret_cast<f32x4*>(p + rows * D + e) = f32x4{dV[ct][4 * r4], dV[ct][4 * r4 + 1], dV[ct][4 * r4 + 2], dV[ct][4 * r4 + 3]};
      }
  };
  if (shares && s < a.sinks) {
    const int slot = sink_job ? a.parts + 2 * part + (w >> 1) : part;
    give(a.sink_part + (((int64_t)bk * (a.parts + 2 * a.far) + slot) * 2 * a.sinks + s) * D, a.sinks);
  } else if (!sink_job && a.parts > 1 && s < s_end) {
    give(a.part + (((int64_t)bk * a.parts + part) * 2 * a.L + s) * D, a.L);
  }
}

// Gradient rows of k or v from their shares [bk][slot][2][n_rows][D].  The first workgroups of a head take a sink's row each, its
// shares dealt out over the threads (they have the longest way); the others several of the other rows.
template <int D>
__global__ __launch_bounds__(256) void window_shares_kernel(WindowArgs a) {
  constexpr int LR = D / 4, PER = 256 / LR;      // threads of a row; rows (or slots) at a time
  __shared__ __attribute__((aligned(16))) float sum[PER][D];
  const int kv = blockIdx.x & 1, bk = blockIdx.x >> 1, b = bk / a.Hkv, hk = bk % a.Hkv;
  const int e = threadIdx.x % LR * 4, u = threadIdx.x / LR;
  const int n_sinks = a.far > 0 ? a.sinks : 0;
  const bool sink = (int)blockIdx.y < n_sinks;
  const int n_rows = sink ? a.sinks : a.L, slots = sink ? a.parts + 2 * a.far : a.parts;
  const int row = sink ? blockIdx.y : (blockIdx.y - n_sinks) * PER + u;
  if (!sink && (row >= a.L || row < n_sinks)) return;
  const int len = clamp_len(a.lens, b, a.L);
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  if (row < len) {
    const float* p = (sink ? a.sink_part : a.part) + (((int64_t)bk * slots * 2 + kv) * n_rows + row) * D + e;
    const int first = sink ? u : 0, step = sink ? PER : 1;
#pragma unroll 4
    for (int i = first; i < slots; i += step) x += *reinterpret_cast<const f32x4*>(p + (int64_t)i * 2 * n_rows * D);
  }
  if (sink) {
    *reinterpret_cast<f32x4*>(&sum[u][e]) = x;
    __syncthreads();
    if (u > 0) return;
#pragma unroll
    for (int i = 1; i < PER; ++i) x += *reinterpret_cast<const f32x4*>(&sum[i][e]);
  }
  if (!kv) x *= a.dk_scale;
  const Rows& o = kv ? a.dv : a.dk;
  uint16_t* out = const_cast<uint16_t*>(static_cast<const uint16_t*>(o.p)) + b * o.b + hk * o.h + row * o.t;
  *reinterpret_cast<u32x2*>(out + e) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
}

template <int D>
hipError_t launch(const WindowArgs& a, hipStream_t s) {
  const int heads = a.B * a.Hkv, tiles = (a.L + 127) / 128;
  hipError_t e = LINATTN_MAX_LDS_ONCE((window_dq_kernel<D>), Cfg<D>::TILES);
  if (e != hipSuccess) return e;
  e = LINATTN_MAX_LDS_ONCE((window_dkv_kernel<D>), Cfg<D>::DKV_BYTES);
  if (e != hipSuccess) return e;
  window_dq_kernel<D><<<dim3((unsigned)xcd_grid(heads, a.H / a.Hkv * tiles)), 256, Cfg<D>::TILES, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  window_dkv_kernel<D><<<dim3((unsigned)xcd_grid(heads, a.far + a.parts * tiles)), 256, Cfg<D>::DKV_BYTES, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int n_sinks = a.far > 0 ? a.sinks : 0, blocks = n_sinks + (a.parts > 1 ? (a.L + 1024 / D - 1) / (1024 / D) : 0);
  if (blocks > 0) {
    window_shares_kernel<D><<<dim3(2 * heads, blocks), 256, 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_window_backward(const WindowArgs& a, int d, hipStream_t s) { return d == 64 ? launch<64>(a, s) : launch<128>(a, s); }

}  // namespace linattn
