// Prefill of linear attention with a decay, fp32 rows, in exact fp32 products (v_mfma_f32_32x32x2_f32); also the three
// products of its gradient.  The mathematics and the ownership are those of decay_prefill.hip in groups of 32 tokens:
// wave w owns the value columns 32w .. 32w+31 and keeps S[:, 32w..] in its accumulators.  An accumulator register is
// itself the operand of the fp32 instruction (rows i and i + 4 in the two halves of the wave), so neither S nor a
// weight is converted or moved.  The 32 x 32 scores of a group are one tile; their contraction is cut over the waves
// and the parts are added where they are read.
//
// Bound: the fp32 matrix rate (about 4 d^2 + 64 d flops a token and head against 16 d bytes).  Measured at 48 padded heads of 64 over
// 1001 tokens, in 8 segments of four groups: 43 us, of which the first pass 13 and the rows 26; 256 heads of 128 over 1000 tokens
// 246 us, 77 TFLOP/s (one wave on every SIMD, whose reads and products take turns).
#include "common.h"
#include "decay.h"
#include "kernels.h"
#include "swizzle.h"

namespace linattn {

namespace {

constexpr int C = 32;

template <int D>
struct Cfg {
  static constexpr int NW = D / 32, NT = 64 * NW;
  static constexpr int RS = D + 4;          // LDS row stride, floats
  static constexpr int PS = C + 4;
  static constexpr int FLOATS = 3 * C * RS + NW * C * PS;
  static constexpr int PPR = D / 4;
  static constexpr int NP = C * PPR / NT;
  static constexpr int RT = D / 32;
};

struct Walk {
  const float* p;
  int64_t t;
};
__device__ __forceinline__ Walk walk(const Rows& r, int b, int h) { return {static_cast<const float*>(r.p) + b * r.b + h * r.h, r.t}; }

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ int acc_row(int r, int hi) { return (r & 3) + 8 * (r >> 2) + 4 * hi; }

template <int D, bool STATE_ONLY>
__global__ __launch_bounds__(Cfg<D>::NT, 1) void decay_prefill_f32_kernel(DecayArgs a) {
  using G = Cfg<D>;
  __shared__ __attribute__((aligned(16))) float smem[G::FLOATS];
  float *Ql = smem, *Kl = Ql + C * G::RS, *Vl = Kl + C * G::RS, *Pl = Vl + C * G::RS;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  // first pass: the pieces of all segments but the last, behind which nothing starts
  const int nseg = STATE_ONLY ? (a.nseg - 1) * a.pieces : a.nseg, seg_len = STATE_ONLY ? a.piece_len : a.seg_len;
  const int seg = blockIdx.x % nseg, bhr = blockIdx.x / nseg;
  const int bh = bhr / a.roles, b = bh / a.H, h = bh % a.H;   // (the roles of a head side by side: they read the same rows)
  const DecayRole& role = a.role[bhr % a.roles];
  const int reverse = role.reverse;
  const Walk wq = walk(role.q, b, h), wk = walk(role.k, b, h), wv = walk(role.v, b, h), wo = walk(role.out, b, h);
  const int len = clamp_len(a.lens, b, a.L);
  const int t_begin = seg * seg_len;
  const int t_end = t_begin + seg_len < a.L ? t_begin + seg_len : a.L;
  const float g2 = decay_log2(a.log_decay, h);
  float* slots = a.ws + (size_t)bhr * a.nseg * a.pieces * (D * D);
  const int c0 = 32 * w;

  f32x16 S[G::RT];
  const float* S0 = STATE_ONLY ? nullptr : a.nseg > 1 && !a.fold ? slots + (size_t)seg * (D * D) : a.S_in ? a.S_in + (size_t)bh * D * D : nullptr;
#pragma unroll
  for (int it = 0; it < G::RT; ++it)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[it][r] = S0 ? S0[(32 * it + acc_row(r, hi)) * D + c0 + l32] : 0.f;

  if (!STATE_ONLY && a.nseg > 1 && a.fold) {
    for (int j = 0; j < seg * a.pieces; ++j) {
      const float* inc = slots + (size_t)j * (D * D);
      const Fade fade(a.log_decay, h, segment_tokens(j, a.piece_len, len));
#pragma unroll
      for (int it = 0; it < G::RT; ++it)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[it][r] = fade.of(S[it][r]) + inc[(32 * it + acc_row(r, hi)) * D + c0 + l32];
    }
  }

  float fp[16], fv[16];                     // of the scores (key acc_row(r), query l32); of the value rows acc_row(r)
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int gap = l32 - acc_row(r, hi);
    fp[r] = gap >= 0 ? decay_pow(g2, gap) * a.scale : 0.f;
    fv[r] = decay_pow(g2, C - 1 - acc_row(r, hi));
  }
  const float fq = decay_pow(g2, l32 + 1) * a.scale;
  const Fade fade32(a.log_decay, h, C);
  const int slow32 = __builtin_amdgcn_readfirstlane(fade32.slow);

  f32x4 rq[G::NP], rk[G::NP], rv[G::NP];
  auto request = [&](int tok0) {
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + G::NT * i, t = tok0 + p / G::PPR, c = p % G::PPR * 4;
      const int row = t < t_end && t < len ? walk_row(t, len, reverse) : 0;
      if (!STATE_ONLY) rq[i] = *reinterpret_cast<const f32x4*>(wq.p + row * wq.t + c);
      rk[i] = *reinterpret_cast<const f32x4*>(wk.p + row * wk.t + c);
      rv[i] = *reinterpret_cast<const f32x4*>(wv.p + row * wv.t + c);
    }
  };
  float* gout = const_cast<float*>(wo.p);

  const int live_end = t_end < len ? t_end : len;
  const int ng = live_end > t_begin ? (live_end - t_begin + C - 1) / C : 0;
  if (ng > 0) request(t_begin);
  for (int gi = 0; gi < ng; ++gi) {
    const int tok0 = t_begin + gi * C;
    const int n = live_end - tok0 < C ? live_end - tok0 : C;
    __syncthreads();                        // every wave is done with the rows of the group before
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + G::NT * i, t = tok0 + p / G::PPR;
      float* d = Ql + p / G::PPR * G::RS + p % G::PPR * 4;
      const bool in = t < live_end;
      const f32x4 z = {0.f, 0.f, 0.f, 0.f};
      if (!STATE_ONLY) *reinterpret_cast<f32x4*>(d) = in ? rq[i] : z;
      *reinterpret_cast<f32x4*>(d + C * G::RS) = in ? rk[i] : z;
      *reinterpret_cast<f32x4*>(d + 2 * C * G::RS) = in ? rv[i] : z;
    }
    __syncthreads();
    if (gi + 1 < ng) request(tok0 + C);

    if (n < C) {                              // (the last group of all: the powers are not needed again)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = acc_row(r, hi);
        fv[r] = i < n ? decay_pow(g2, n - 1 - i) : 0.f;
      }
    }
    f32x16 O = {};
    if (!STATE_ONLY) {
      // ---- this wave's part of P^T: 32 features, of which a half of the wave takes 16
      f32x16 x = {};
#pragma unroll
      for (int f = 0; f < 16; f += 4) {
        const f32x4 kk = *reinterpret_cast<const f32x4*>(Kl + l32 * G::RS + c0 + 16 * hi + f);
        const f32x4 qq = *reinterpret_cast<const f32x4*>(Ql + l32 * G::RS + c0 + 16 * hi + f);
#pragma unroll
        for (int i = 0; i < 4; ++i) x = mfma_f32(kk[i], qq[i], x);
      }
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 y = {x[4 * r4], x[4 * r4 + 1], x[4 * r4 + 2], x[4 * r4 + 3]};
        *reinterpret_cast<f32x4*>(Pl + (w * C + l32) * G::PS + 8 * r4 + 4 * hi) = y;
      }
      // ---- S^T Q^T
#pragma unroll
      for (int it = 0; it < G::RT; ++it)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4 qq = *reinterpret_cast<const f32x4*>(Ql + l32 * G::RS + 32 * it + 8 * r4 + 4 * hi);
#pragma unroll
          for (int i = 0; i < 4; ++i) O = mfma_f32(S[it][4 * r4 + i], qq[i], O);
        }
      O *= fq;
    }
    float v[16];                            // V[acc_row(r)][c0 + l32]
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = Vl[acc_row(r, hi) * G::RS + c0 + l32];
    if (n < C) {
      const Fade fade(a.log_decay, h, n);
#pragma unroll
      for (int it = 0; it < G::RT; ++it)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[it][r] = fade.of(S[it][r]);
    } else if (slow32) {
#pragma unroll
      for (int it = 0; it < G::RT; ++it) S[it] += S[it] * fade32.f;
    } else {
#pragma unroll
      for (int it = 0; it < G::RT; ++it) S[it] *= fade32.f;
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int it = 0; it < G::RT; ++it) S[it] = mfma_f32(Kl[acc_row(r, hi) * G::RS + 32 * it + l32], v[r] * fv[r], S[it]);
    read_ahead<8, 1, 1, 16 * G::RT>();
    if (!STATE_ONLY) {
      __syncthreads();                      // the parts of P; every wave is done with the Q rows
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < G::NW; ++u) p += *reinterpret_cast<const f32x4*>(Pl + (u * C + l32) * G::PS + 8 * r4 + 4 * hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) O = mfma_f32(v[4 * r4 + i], fp[4 * r4 + i] != 0.f ? p[i] * fp[4 * r4 + i] : 0.f, O);
      }
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 y = {O[4 * r4], O[4 * r4 + 1], O[4 * r4 + 2], O[4 * r4 + 3]};
        *reinterpret_cast<f32x4*>(Ql + l32 * G::RS + c0 + 8 * r4 + 4 * hi) = y;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < G::NP; ++i) {
        const int p = tid + G::NT * i, t = tok0 + p / G::PPR;
        if (t < t_end) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(Ql + p / G::PPR * G::RS + p % G::PPR * 4), z = {0.f, 0.f, 0.f, 0.f};
          *reinterpret_cast<f32x4*>(gout + walk_row(t, len, reverse) * wo.t + p % G::PPR * 4) = t < len ? x : z;
        }
      }
    }
  }
  if (!STATE_ONLY) {
    for (int e = tid; e < (t_end - t_begin - ng * C) * G::PPR; e += G::NT) {
      const f32x4 z = {0.f, 0.f, 0.f, 0.f};
      *reinterpret_cast<f32x4*>(gout + (int64_t)(t_begin + ng * C + e / G::PPR) * wo.t + e % G::PPR * 4) = z;
    }
  }
  float* So = STATE_ONLY ? slots + (size_t)seg * (D * D) : a.S_out && seg == a.nseg - 1 ? a.S_out + (size_t)bh * D * D : nullptr;
  if (So) {
#pragma unroll
    for (int it = 0; it < G::RT; ++it)
#pragma unroll
      for (int r = 0; r < 16; ++r) So[(32 * it + acc_row(r, hi)) * D + c0 + l32] = S[it][r];
  }
}

template <int D, bool STATE_ONLY>
hipError_t launch(const DecayArgs& a, hipStream_t s) {
  decay_prefill_f32_kernel<D, STATE_ONLY><<<dim3(a.roles * a.B * a.H * (STATE_ONLY ? (a.nseg - 1) * a.pieces : a.nseg)), Cfg<D>::NT, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decay_first_pass_f32(const DecayArgs& a, int d, hipStream_t s) { return d == 64 ? launch<64, true>(a, s) : launch<128, true>(a, s); }
hipError_t launch_decay_rows_f32(const DecayArgs& a, int d, hipStream_t s) { return d == 64 ? launch<64, false>(a, s) : launch<128, false>(a, s); }

}  // namespace linattn
