// Softmax attention over a sliding window with sinks, bf16 rows, on the matrix cores.
//
//   out_t = sum_s p_ts v_s / sum_s p_ts,   p_ts = exp(scale q_t.k_s - m_t),   s <= t and (s > t - window or s < sinks)
//
// One pass over the visible keys with a running maximum m and a running sum.  A workgroup takes 128 queries of a head,
// a wave 32 of them; 64 or 32 keys at a time lie in one of two LDS buffers while the next are on their way into the other.
// S^T = K Q^T with the keys in the accumulator's rows and a query per lane, so a query's statistics are a lane's own
// (and its partner's 32 lanes on), and the weights, packed to bf16, are the operand of O^T += V^T P^T as they stand: the
// accumulator layout is the operand layout up to a permutation of the keys, which is applied to the transposed reads of
// V.  Key tiles that no query of the tile sees are not visited; masks are computed only where a border crosses.
//
// The weights are rounded to bf16 once for their product with V (not in the sum that divides it): out is off by 2.2e-3 in the 2-norm, of
// which its own rounding is 1.6e-3.  In two terms the first part goes, for a third more time (530 -> 700 us at the size below).
//
// Bound: the matrix cores (4 d flops a visible pair; 53 % of the cycles) beside the vector ALUs (some 190 instructions for 32 products
// of a wave, 32 of them exponentials; 49 %), at 1.8 GHz (power).  Measured at 64 heads of 128 over 8192 tokens, a window of 2048: 505 to 525 us
// (boards differ), 940 TFLOP/s of 1361 that a large library product reaches.
#include "common.h"
#include "kernels.h"
#include "mfma_util.h"
#include "window.h"

namespace linattn {

namespace {

constexpr int QT = 128;                         // queries of a workgroup; KT: keys at a time

constexpr float kLate = 8.f;   // log2: how far a running maximum may lie behind before the sums are scaled anew

template <int D, int KT>
struct Cfg {
  static constexpr int BUF = 2 * KT * D;        // elements: K, V
  static constexpr int OS = D + 8;              // finished rows
  static constexpr int BYTES = (2 * BUF > QT * OS ? 2 * BUF : QT * OS) * 2;
  static constexpr int PPR = D / 8;
};

template <int D, int KT>
__global__ __launch_bounds__(256, KT == 32 ? 3 : 2) void window_prefill_kernel(WindowArgs a) {
  using G = Cfg<D, KT>;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  // the query heads that share keys side by side, then the query tiles
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
  uint16_t* gout = const_cast<uint16_t*>(static_cast<const uint16_t*>(a.out.p)) + b * a.out.b + h * a.out.h;
  float* glse = a.lse ? a.lse + ((int64_t)b * a.H + h) * a.L : nullptr;
  if (t0 >= len) {                              // behind the end of the sequence
    for (int e = tid; e < (t_end - t0) * G::PPR; e += 256) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      *reinterpret_cast<u32x4*>(gout + (t0 + e / G::PPR) * a.out.t + e % G::PPR * 8) = z;
    }
    if (glse)
      for (int t = t0 + tid; t < t_end; t += 256) glse[t] = -__builtin_inff();
    return;
  }
  const uint16_t* gq = static_cast<const uint16_t*>(a.q.p) + b * a.q.b + h * a.q.h;
  const uint16_t* gk = static_cast<const uint16_t*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const uint16_t* gv = static_cast<const uint16_t*>(a.v.p) + b * a.v.b + hk * a.v.h;
  const float c = window_log2_scale(a.scale);
  constexpr int KS = D / 16, CT = D / 32, NS = KT / 32 * KS, NP = KT / 16 * CT, AHEAD = KT == 32 ? 2 : D == 128 ? 6 : 3;
  const Swizzled<D> lds(lane, 4);

  const int t = t0 + 32 * w + l32;              // this lane's query
  const int tw = t0 + 32 * w;                   // the wave's first
  bf16x8 qop[D / 16];
  {
    const uint16_t* p = gq + (t < len ? t : len - 1) * a.q.t + 8 * hi;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qop[ks] = *reinterpret_cast<const bf16x8*>(p + 16 * ks);
  }
  // key tiles: those of the sinks that lie before the window's, then the window's
  const int last = (t_end < len ? t_end : len) - 1;
  const int lo = (t0 - a.window + 1 > 0 ? t0 - a.window + 1 : 0) / KT;
  const int sink_tiles = (a.sinks + KT - 1) / KT, ns = sink_tiles < lo ? sink_tiles : lo;
  const int nk = ns + last / KT - lo + 1;
  auto key0 = [&](int i) { return (i < ns ? i : lo + i - ns) * KT; };

  const Fetch<D, KT> fetch(tid);
  auto request = [&](int i, uint16_t* buf) {
    const int s0 = key0(i);
    fetch.request(buf, gk + s0 * a.k.t, a.k.t, len - s0);
    fetch.request(buf + KT * D, gv + s0 * a.v.t, a.v.t, len - s0);
  };
  auto arrive = [&](int i, uint16_t* buf) {     // ... and, behind the barrier, everybody's
    const int n = len - key0(i);
    fetch.arrived();
    fetch.trim(buf, n, tid);
    fetch.trim(buf + KT * D, n, tid);
    __syncthreads();
  };

  f32x16 O[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) O[i] = f32x16{};
  float m = -__builtin_inff(), l = 0.f;         // l: this lane's half of the keys

  auto tile_of = [&](int i, const uint16_t* Kl) {
    const uint16_t* Vl = Kl + KT * D;
    const int s0 = key0(i);
    if (!(s0 <= tw + 31 && (s0 + KT - 1 > tw - a.window || s0 < a.sinks))) return;
    // the matrix operands in the order of their use, AHEAD of them read before they are needed
    bf16x8 op[NS + NP];
    auto read = [&](int i) {
      if (i < NS) op[i] = lds.rows(Kl, 32 * (i / KS), i % KS);
      else if (i < NS + NP) op[i] = lds.cols_acc(Vl, 16 * ((i - NS) / CT), (i - NS) % CT);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read(i);
    __builtin_amdgcn_sched_barrier(0);
    f32x16 x[KT / 32] = {};
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      x[i / KS] = mfma(op[i], qop[i % KS], x[i / KS]);
      read(i + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
    }
    const bool all = s0 + KT - 1 <= tw && (s0 > tw + 31 - a.window || s0 + KT <= a.sinks);
    if (!all) {
#pragma unroll
      for (int kt = 0; kt < KT / 32; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!window_sees(t, s0 + 32 * kt + acc_row(r, hi), a.window, a.sinks)) x[kt][r] = -__builtin_inff();
    }
    float top = x[0][0];
#pragma unroll
    for (int kt = 0; kt < KT / 32; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, x[kt][r]);
    top = max_xor32(top) * c;
    if (__any(top > m + kLate)) {
      const float m2 = fmaxf(m, top);
      const float f = m2 == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      l *= f;
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct) O[ct] *= f;
    }
    const float mm = m == -__builtin_inff() ? 0.f : m;         // nothing seen yet: every weight is exp2(-inf)
    auto weigh = [&](int j, int from, int to) {                // 16 keys: eight of this lane
#pragma unroll
      for (int r = from; r < to; ++r) {
        const int i = 8 * (j % 2) + r;
        x[j / 2][i] = __builtin_amdgcn_exp2f(x[j / 2][i] * c - mm);
        l += x[j / 2][i];
      }
    };
    weigh(0, 0, 8);
#pragma unroll
    for (int j = 0; j < KT / 16; ++j) {
      const bf16x8 p = pack8(x[j / 2], 8 * (j % 2));
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        __builtin_amdgcn_sched_barrier(0);
        O[ct] = mfma(op[NS + CT * j + ct], p, O[ct]);
        read(NS + CT * j + ct + AHEAD);
        if (j + 1 < KT / 16) weigh(j + 1, 8 * ct / CT, 8 * (ct + 1) / CT);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto turn = [&](int i, uint16_t* __restrict cur, uint16_t* __restrict next) {   // (see Fetch)
    arrive(i, cur);
    if (i + 1 < nk) request(i + 1, next);
    tile_of(i, cur);
  };
  uint16_t *even = smem, *odd = smem + G::BUF;
  request(0, even);
  for (int i = 0; i < nk; i += 2) {             // (two at a time: the buffers' addresses are constants)
    turn(i, even, odd);
    if (i + 1 < nk) turn(i + 1, odd, even);
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
      u32x2 y = {pack_bf16x2(O[ct][4 * r4] * inv, O[ct][4 * r4 + 1] * inv), pack_bf16x2(O[ct][4 * r4 + 2] * inv, O[ct][4 * r4 + 3] * inv)};
      *reinterpret_cast<u32x2*>(smem + (32 * w + l32) * G::OS + 32 * ct + 8 * r4 + 4 * hi) = y;
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < QT * G::PPR / 256; ++i) {
    const int p = tid + 256 * i, r = p / G::PPR;
    const u32x4 x = *reinterpret_cast<const u32x4*>(smem + r * G::OS + p % G::PPR * 8), z = {0u, 0u, 0u, 0u};
    if (t0 + r < t_end) *reinterpret_cast<u32x4*>(gout + (t0 + r) * a.out.t + p % G::PPR * 8) = t0 + r < len ? x : z;
  }
}

template <int D, int KT>
hipError_t launch(const WindowArgs& a, int64_t grid, hipStream_t s) {
  hipError_t e = LINATTN_MAX_LDS_ONCE((window_prefill_kernel<D, KT>), (Cfg<D, KT>::BYTES));
  if (e != hipSuccess) return e;
  window_prefill_kernel<D, KT><<<dim3((unsigned)grid), 256, Cfg<D, KT>::BYTES, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_window_prefill_bf16(const WindowArgs& a, int d, hipStream_t s) {
  const int64_t grid = xcd_grid(a.B * a.Hkv, a.H / a.Hkv * ((a.L + QT - 1) / QT));
  if (d == 64) return launch<64, 64>(a, grid, s);
  // 32 keys at a time leave room for three workgroups on a compute unit, where there are as many: 540 -> 524 us at the size above.
  // Where there are fewer a wave is alone with what it waits for, twice as often: 151 -> 211 us at 4 heads over 8192 tokens.
  return grid >= 3 * 256 ? launch<128, 32>(a, grid, s) : launch<128, 64>(a, grid, s);
}

}  // namespace linattn
