// Prefill of linear attention with a decay, bf16 rows, on the matrix cores; also the three products of its gradient.
//
//   out_t = scale sum_{s<=t} lambda^{t-s} (q_t.k_s) v_s
//
// in groups of 64 tokens: with S the state before a group, i = 0..63 a token's place in it and n the tokens it has,
//
//   O^T  = lambda^{i+1} (S^T Q^T) + V^T P^T,     P_ij = lambda^{i-j} (q_i.k_j) for j <= i
//   S   <- lambda^n S + K^T V',                  v'_j = lambda^{n-1-j} v_j
//
// Every power has an exponent >= 0, so nothing overflows however fast a head forgets.  One workgroup walks one head (or
// a segment of it); wave w owns the value columns 32w .. 32w+31: S[:, 32w..] stays in its accumulators, and is its own
// MFMA operand for the read-out (the accumulator layout is the operand layout up to a permutation of the contraction
// index, which is applied to Q's LDS address).  The rows are requested one group ahead into registers and go to one of
// two LDS buffers; the finished rows go back through the Q rows of their own buffer, so that whole rows are stored.
// V' enters the state as the sum of two bf16 terms (sixteen significant bits: S is handed back in fp32 and lives on in
// generation); where the state is only this launch's own (the gradient) one term is enough.
//
// The gradient is the same function with other roles: dq = F(dout, v, k), and over reversed time dk = F(v, dout, q),
// dv = F(k, q, dout); a launch carries up to three roles.
//
// Bound: HBM (8 d bytes a token and head: at d = 128 1 KB, against 82 K flops).
#include "common.h"
#include "decay.h"
#include "kernels.h"
#include "mfma_util.h"

namespace linattn {

namespace {

constexpr int C = 64;                       // tokens per group

template <int D>
struct Cfg {
  static constexpr int NW = D / 32, NT = 64 * NW;
  static constexpr int RS = D + 16;         // LDS row stride
  static constexpr int PS = C + 8;
  static constexpr int BUF = 3 * C * RS;    // elements of one buffer: Q, K, V
  static constexpr int BYTES = (2 * BUF + C * PS) * 2;
  static constexpr int PPR = D / 8;         // 16-byte pieces per row
  static constexpr int NP = C * PPR / NT;   // pieces per thread and tensor
  static constexpr int RT = D / 32;         // 32-row tiles of S
  static constexpr int TW = (3 + NW - 1) / NW;   // score tiles per wave
};

struct Walk {                               // where one tensor's rows of this (b, h) are
  const uint16_t* p;
  int64_t t;
};
__device__ __forceinline__ Walk walk(const Rows& r, int b, int h) {
  return {static_cast<const uint16_t*>(r.p) + b * r.b + h * r.h, r.t};
}

template <int D, bool STATE_ONLY, bool TWO>
__global__ __launch_bounds__(Cfg<D>::NT, 1) void decay_prefill_kernel(DecayArgs a) {
  using G = Cfg<D>;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  uint16_t* Pl = smem + 2 * G::BUF;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int seg = blockIdx.x % a.nseg, bhr = blockIdx.x / a.nseg;
  const int bh = bhr / a.roles, b = bh / a.H, h = bh % a.H;   // (the roles of a head side by side: they read the same rows)
  const DecayRole& role = a.role[bhr % a.roles];
  const int reverse = role.reverse;
  const Walk wq = walk(role.q, b, h), wk = walk(role.k, b, h), wv = walk(role.v, b, h), wo = walk(role.out, b, h);
  const int len = clamp_len(a.lens, b, a.L);
  const int t_begin = seg * a.seg_len;
  const int t_end = t_begin + a.seg_len < a.L ? t_begin + a.seg_len : a.L;
  const float g2 = decay_log2(a.log_decay, h);
  float* slot = a.ws + ((size_t)bhr * a.nseg + seg) * (D * D);
  if (STATE_ONLY && seg == a.nseg - 1) return;   // nothing starts behind the last segment
  const int c0 = 32 * w;

  // ---- the state's 32 columns: row (r&3) + 8(r>>2) + 4hi of tile it, column c0 + l32
  f32x16 S[G::RT];
  const float* S0 = STATE_ONLY ? nullptr : a.nseg > 1 ? slot : a.S_in ? a.S_in + (size_t)bh * D * D : nullptr;
#pragma unroll
  for (int it = 0; it < G::RT; ++it)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[it][r] = S0 ? S0[(32 * it + (r & 3) + 8 * (r >> 2) + 4 * hi) * D + c0 + l32] : 0.f;

  // ---- powers of the decay that every whole group uses
  f32x16 fac[G::TW];                        // this wave's score tiles: number w, w + NW, .. of (0,0), (1,0), (1,1)
#pragma unroll
  for (int i = 0; i < G::TW; ++i) {
    const int n = w + i * G::NW, tt = n > 0, st = n > 1;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int gap = 32 * (tt - st) + l32 - ((r & 3) + 8 * (r >> 2) + 4 * hi);
      fac[i][r] = gap >= 0 ? decay_pow(g2, gap) : 0.f;
    }
  }
  const float fq0 = decay_pow(g2, l32 + 1) * a.scale, fq1 = decay_pow(g2, l32 + 33) * a.scale;
  float fv[4][8];                           // of the rows 16ks + 8hi + j of a group
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int j = 0; j < 8; ++j) fv[ks][j] = decay_pow(g2, 63 - (16 * ks + 8 * hi + j));

  u32x4 rq[G::NP], rk[G::NP], rv[G::NP];
  auto request = [&](int tok0) {            // rows past the end re-read row 0; they are dropped in put()
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + G::NT * i, t = tok0 + p / G::PPR, c = p % G::PPR * 8;
      const int row = t < t_end && t < len ? walk_row(t, len, reverse) : 0;
      if (!STATE_ONLY) rq[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(wq.p + row * wq.t + c));
      rk[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(wk.p + row * wk.t + c));
      rv[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(wv.p + row * wv.t + c));
    }
  };
  auto put = [&](int tok0, uint16_t* buf) {
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + G::NT * i, t = tok0 + p / G::PPR;
      uint16_t* d = buf + p / G::PPR * G::RS + p % G::PPR * 8;
      const bool in = t < t_end && t < len;
      const u32x4 z = {0u, 0u, 0u, 0u};
      if (!STATE_ONLY) *reinterpret_cast<u32x4*>(d) = in ? rq[i] : z;
      *reinterpret_cast<u32x4*>(d + C * G::RS) = in ? rk[i] : z;
      *reinterpret_cast<u32x4*>(d + 2 * C * G::RS) = in ? rv[i] : z;
    }
  };
  uint16_t* gout = const_cast<uint16_t*>(wo.p);
  auto store_rows = [&](int tok0, const uint16_t* buf) {
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + G::NT * i, t = tok0 + p / G::PPR;
      if (t < t_end) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(buf + p / G::PPR * G::RS + p % G::PPR * 8), z = {0u, 0u, 0u, 0u};
        __builtin_nontemporal_store(t < len ? x : z, reinterpret_cast<u32x4*>(gout + walk_row(t, len, reverse) * wo.t + p % G::PPR * 8));
      }
    }
  };

  const int live_end = t_end < len ? t_end : len;                       // tokens that are there
  const int ng = live_end > t_begin ? (live_end - t_begin + C - 1) / C : 0;
  if (ng > 0) {
    request(t_begin);
    put(t_begin, smem);
  }
  for (int gi = 0; gi < ng; ++gi) {
    const int tok0 = t_begin + gi * C;
    uint16_t* buf = smem + (gi & 1) * G::BUF;
    uint16_t *Ql = buf, *Kl = buf + C * G::RS, *Vl = buf + 2 * C * G::RS;
    const int n = live_end - tok0 < C ? live_end - tok0 : C;
    __syncthreads();                        // the group's rows, and the finished rows of the group before
    if (gi + 1 < ng) request(tok0 + C);
    if (!STATE_ONLY && gi > 0) store_rows(tok0 - C, smem + ((gi + 1) & 1) * G::BUF);

    bf16x8 vop[4];                          // V[16ks + 8hi + 0..7][c0 + l32]
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) vop[ks] = tr_operand(Vl, G::RS, 16 * ks, c0, lane);

    f32x16 O[2];
    if (!STATE_ONLY) {
      // ---- this wave's tiles of P^T, weighted
#pragma unroll
      for (int i = 0; i < G::TW; ++i) {
        const int nt = w + i * G::NW, tt = nt > 0, st = nt > 1;
        if (nt < 3) {
          f32x16 x = {};
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
            x = mfma(lds_row8(Kl + (32 * st + l32) * G::RS + 16 * ks + 8 * hi), lds_row8(Ql + (32 * tt + l32) * G::RS + 16 * ks + 8 * hi), x);
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = fac[i][r] != 0.f ? x[r] * fac[i][r] * a.scale : 0.f;
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const u32x2 y = {pack_bf16x2(x[4 * r4], x[4 * r4 + 1]), pack_bf16x2(x[4 * r4 + 2], x[4 * r4 + 3])};
            *reinterpret_cast<u32x2*>(Pl + (32 * tt + l32) * G::PS + 32 * st + 8 * r4 + 4 * hi) = y;
          }
        }
      }
      // ---- S^T Q^T
      O[0] = f32x16{}; O[1] = f32x16{};
#pragma unroll
      for (int it = 0; it < G::RT; ++it)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const bf16x8 s = pack8(S[it], 8 * half);
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            const uint16_t* q = Ql + (32 * tt + l32) * G::RS + 32 * it + 16 * half + 4 * hi;
            O[tt] = mfma(s, cat4(lds_row4(q), lds_row4(q + 8)), O[tt]);
          }
        }
      O[0] *= fq0; O[1] *= fq1;
    }
    // ---- the state takes the group
    const float keep = decay_pow(g2, n);
#pragma unroll
    for (int it = 0; it < G::RT; ++it) S[it] *= keep;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      f32x16 x;                             // eight values; split8 and pack8 take them from an accumulator
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = 16 * ks + 8 * hi + j;
        const float f = n == C ? fv[ks][j] : i < n ? decay_pow(g2, n - 1 - i) : 0.f;
        x[j] = (float)vop[ks][j] * f;
      }
      bf16x8 vh, vo;
      if (TWO) split8(x, 0, vh, vo);
      else vh = pack8(x, 0);
#pragma unroll
      for (int it = 0; it < G::RT; ++it) {
        const bf16x8 k = tr_operand(Kl, G::RS, 16 * ks, 32 * it, lane);
        S[it] = mfma(k, vh, S[it]);
        if (TWO) S[it] = mfma(k, vo, S[it]);
      }
    }
    if (!STATE_ONLY) {
      __syncthreads();                      // P; and every wave is done with the Q rows
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
        for (int ks = 0; ks < 2 * (tt + 1); ++ks)
          O[tt] = mfma(vop[ks], lds_row8(Pl + (32 * tt + l32) * G::PS + 16 * ks + 8 * hi), O[tt]);
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const u32x2 y = {pack_bf16x2(O[tt][4 * r4], O[tt][4 * r4 + 1]), pack_bf16x2(O[tt][4 * r4 + 2], O[tt][4 * r4 + 3])};
          *reinterpret_cast<u32x2*>(Ql + (32 * tt + l32) * G::RS + c0 + 8 * r4 + 4 * hi) = y;
        }
      }
    }
    if (gi + 1 < ng) put(tok0 + C, smem + ((gi + 1) & 1) * G::BUF);
  }
  if (!STATE_ONLY) {
    if (ng > 0) {
      __syncthreads();
      store_rows(t_begin + (ng - 1) * C, smem + ((ng - 1) & 1) * G::BUF);
    }
    // rows behind the end of the sequence, in groups that the walk has not met
    for (int e = tid; e < (t_end - t_begin - ng * C) * G::PPR; e += G::NT) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      *reinterpret_cast<u32x4*>(gout + (int64_t)(t_begin + ng * C + e / G::PPR) * wo.t + e % G::PPR * 8) = z;
    }
  }
  float* So = STATE_ONLY ? slot : a.S_out && seg == a.nseg - 1 ? a.S_out + (size_t)bh * D * D : nullptr;
  if (So) {
#pragma unroll
    for (int it = 0; it < G::RT; ++it)
#pragma unroll
      for (int r = 0; r < 16; ++r) So[(32 * it + (r & 3) + 8 * (r >> 2) + 4 * hi) * D + c0 + l32] = S[it][r];
  }
}

template <int D, bool STATE_ONLY, bool TWO>
hipError_t launch(const DecayArgs& a, hipStream_t s) {
  using G = Cfg<D>;
  hipError_t e = LINATTN_MAX_LDS_ONCE((decay_prefill_kernel<D, STATE_ONLY, TWO>), G::BYTES);
  if (e != hipSuccess) return e;
  decay_prefill_kernel<D, STATE_ONLY, TWO><<<dim3(a.roles * a.B * a.H * a.nseg), G::NT, G::BYTES, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decay_first_pass_bf16(const DecayArgs& a, int d, hipStream_t s) {
  if (d == 64) return a.exact_state ? launch<64, true, true>(a, s) : launch<64, true, false>(a, s);
  return a.exact_state ? launch<128, true, true>(a, s) : launch<128, true, false>(a, s);
}
hipError_t launch_decay_rows_bf16(const DecayArgs& a, int d, hipStream_t s) {
  if (d == 64) return a.exact_state ? launch<64, false, true>(a, s) : launch<64, false, false>(a, s);
  return a.exact_state ? launch<128, false, true>(a, s) : launch<128, false, false>(a, s);
}

}  // namespace linattn
