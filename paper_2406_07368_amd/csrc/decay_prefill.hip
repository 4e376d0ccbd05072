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
// a segment of it), two waves on every SIMD.  Wave (ct, half) owns the value columns 32ct .. 32ct+31 and one half of S's rows
// for the state, and one half of the group's tokens for the outputs: S[half, 32ct..] stays in its accumulators and, packed, is
// the MFMA operand of the read-out as it stands (the rows' order in the accumulators is made so by the order in which K is
// read); it reads for all 64 tokens and gives the other wave of the pair, through LDS, what that one's tokens get from its
// rows.  The scores are ten 16 x 16 tiles, dealt out over the waves.  Rows come straight into one of two LDS buffers while
// the other is worked on (swizzle.h); finished rows leave through LDS, so that whole rows are stored.
// V' enters the state as the sum of TERMS bf16 terms.  Two carry sixteen significant bits: with one, the gradient's error was
// 1.65 times that of the final rounding alone, with two it is 1.4 times.  A state that is handed back in fp32 takes three, all
// of an fp32 product's bits (its error at LLaMA size: 3.6e-7, with two terms 2.5e-6, for 264 us in the place of 240).
// The weights P and, for its read-out, the state are rounded to bf16 once: the outputs are off by 2.34e-3 in the 2-norm, of which their
// own rounding is 1.66e-3.  The read-out in two terms: 1.79e-3, for 12 % more time (275 -> 306 us, the gradient of the training
// batch 315 -> 364), which these kernels, bound by the issue of instructions, do not have.
//
// The gradient is the same function with other roles: dq = F(dout, v, k), and over reversed time dk = F(v, dout, q),
// dv = F(k, q, dout); a launch carries up to three roles.
//
// HBM is the floor (8 d bytes a token and head: at d = 128 1 KB, against 82 K flops), and what bounds it now is the issue of vector
// and matrix instructions at the clock that the power limit leaves (2.0 GHz).  Measured at 256 heads of 128 over 4096 tokens: 236 us with
// two terms, 264 with three (1.07 GB of rows: 4.5 and 4.1 TB/s; a copy runs at 5.1).
#include "common.h"
#include "decay.h"
#include "kernels.h"
#include "swizzle.h"

namespace linattn {

namespace {

constexpr int C = 64;                       // tokens per group

template <int D>
struct Cfg {
  static constexpr int NW = D / 16, NT = 64 * NW;
  static constexpr int CT = D / 32;              // column tiles of S: the waves 0 .. CT-1 have its upper rows, the others its lower
  static constexpr int IT = D / 64;              // 32-row tiles of a wave's S
  static constexpr int TILE = C * D;             // elements of one tensor's rows
  static constexpr int PPR = D / 8;
  static constexpr int NP = C * PPR / NT;        // 16-byte pieces of a tensor's rows per thread
  static constexpr int TW = (10 + NW - 1) / NW;  // score tiles per wave
  // bytes: two buffers of K, V (, Q); P; what the waves of a pair give each other; finished rows
  static constexpr int KV = 4 * TILE * 2;
  static constexpr int OFF_P = 6 * TILE * 2, OFF_X = OFF_P + C * C * 2, OFF_O = OFF_X + NW * 1024 * 4, ALL = OFF_O + TILE * 2;
};

struct Walk {                                    // one tensor's rows of this (b, h)
  const uint16_t* p;
  int64_t t;
};
__device__ __forceinline__ Walk walk(const Rows& r, int b, int h) {
  return {static_cast<const uint16_t*>(r.p) + b * r.b + h * r.h, r.t};
}

template <int D, bool STATE_ONLY, int TERMS>
__global__ __launch_bounds__(Cfg<D>::NT, 2) void decay_prefill_kernel(DecayArgs a) {
  using G = Cfg<D>;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  uint16_t* Pl = smem + G::OFF_P / 2;
  float* Xl = reinterpret_cast<float*>(smem + G::OFF_X / 2);
  uint16_t* Ol = smem + G::OFF_O / 2;
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), ct = w % G::CT, half = w / G::CT;
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5, l16 = lane & 15, q4 = lane >> 4;
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

  const int live_end = t_end < len ? t_end : len;                        // tokens that are there
  const int ng = live_end > t_begin ? (live_end - t_begin + C - 1) / C : 0;
  const Fetch<D, C, G::NT> fetch(tid);
  uint16_t *even = smem, *odd = smem + (STATE_ONLY ? 2 : 3) * G::TILE;   // K, V, Q
  auto request = [&](int gi, uint16_t* buf) {
    const int tok0 = t_begin + gi * C, n = live_end - tok0;
    auto one = [&](uint16_t* to, const Walk& from) {
      if (reverse) fetch.template request<true>(to, from.p + (int64_t)(len - tok0 - (n < C ? n : C)) * from.t, from.t, n);
      else fetch.request(to, from.p + (int64_t)tok0 * from.t, from.t, n);
    };
    one(buf, wk);
    one(buf + G::TILE, wv);
    if (!STATE_ONLY) one(buf + 2 * G::TILE, wq);
  };
  auto arrive = [&](int gi, uint16_t* buf) {
    const int n = live_end - (t_begin + gi * C);
    fetch.arrived();
    fetch.trim(buf, n, tid);
    fetch.trim(buf + G::TILE, n, tid);
    if (!STATE_ONLY) fetch.trim(buf + 2 * G::TILE, n, tid);
    __syncthreads();
  };
  if (ng > 0) request(0, even);

  // ---- this wave's part of the state: register r of tile it is row 32 (G::IT half + it) + row_of(r), column 32 ct + l32
  auto row_of = [&](int r) { return 16 * (r >> 3) + 8 * hi + (r & 7); };
  auto at = [&](int it, int r) { return (32 * (G::IT * half + it) + row_of(r)) * D + 32 * ct + l32; };
  f32x16 S[G::IT];
  const float* S0 = STATE_ONLY ? nullptr : a.nseg > 1 && !a.fold ? slots + (size_t)seg * (D * D) : a.S_in ? a.S_in + (size_t)bh * D * D : nullptr;
#pragma unroll
  for (int it = 0; it < G::IT; ++it)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[it][r] = S0 ? S0[at(it, r)] : 0.f;
  if (!STATE_ONLY && a.nseg > 1 && a.fold) {     // few segments: what those before this one add, instead of a launch that sums it up
    for (int j = 0; j < seg * a.pieces; ++j) {              // (four increments in flight at once: 40 registers spilled, 8 % slower)
      const float* inc = slots + (size_t)j * (D * D);
      const Fade fade(a.log_decay, h, segment_tokens(j, a.piece_len, len));
#pragma unroll
      for (int it = 0; it < G::IT; ++it)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[it][r] = fade.of(S[it][r]) + inc[at(it, r)];
    }
  }

  // ---- powers of the decay that every whole group uses
  // score tile n of 10: (tb, sb) with sb <= tb; a lane has query 16 tb + l16 and keys 16 sb + 4 q4 + 0..3
  auto tile_row = [](int n) { return n >= 6 ? 3 : n >= 3 ? 2 : n >= 1 ? 1 : 0; };
  f32x4 fac[G::TW];
#pragma unroll
  for (int i = 0; i < G::TW; ++i) {
    const int n = w + i * G::NW, tb = tile_row(n), sb = n - tb * (tb + 1) / 2;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int gap = 16 * (tb - sb) + l16 - (4 * q4 + r);
      fac[i][r] = gap >= 0 ? decay_pow(g2, gap) * a.scale : 0.f;
    }
  }
  const float fq = decay_pow(g2, 32 * half + l32 + 1) * a.scale;         // of this wave's queries
  float fv[4][8];                                                        // of the rows 16ks + 8hi + j of a group
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int j = 0; j < 8; ++j) fv[ks][j] = decay_pow(g2, 63 - (16 * ks + 8 * hi + j));

  const Fade fade64(a.log_decay, h, C);
  const int slow64 = __builtin_amdgcn_readfirstlane(fade64.slow);
  uint16_t* gout = const_cast<uint16_t*>(wo.p);
  auto store_rows = [&](int gi, const uint16_t* Ol) {
    const int tok0 = t_begin + gi * C;
#pragma unroll
    for (int i = 0; i < G::NP; ++i) {
      const int p = tid + G::NT * i, t = tok0 + p / G::PPR;
      if (t < t_end) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(Ol + Swizzled<D>::piece(p / G::PPR, p % G::PPR)), z = {0u, 0u, 0u, 0u};
        __builtin_nontemporal_store(t < len ? x : z, reinterpret_cast<u32x4*>(gout + walk_row(t, len, reverse) * wo.t + p % G::PPR * 8));
      }
    }
  };
  // the tiles of P that are read but hold only later keys, (0, 1) and (2, 3), stay zeros
  if (!STATE_ONLY)
    for (int i = tid; i < C * C / 8; i += G::NT) *reinterpret_cast<u32x4*>(Pl + 8 * i) = u32x4{0u, 0u, 0u, 0u};
  const Swizzled<D> kv0(lane, 8), kx0(lane, 8, true);
  const Swizzled<C> pr(lane, 8);
  const int tile16 = Swizzled<D>::piece(l16, D / 32 * q4);   // a lane's piece of a 16-row operand; its ks-th: ^ (ks << 3)

  auto group = [&](int gi, uint16_t* __restrict cur, uint16_t* __restrict next, uint16_t* __restrict Pl, float* __restrict Xl, uint16_t* __restrict Ol) {
    const int tok0 = t_begin + gi * C;
    const uint16_t *Kl = cur, *Vl = Kl + G::TILE, *Ql = Vl + G::TILE;
    const int n = live_end - tok0 < C ? live_end - tok0 : C;
    arrive(gi, cur);                             // the group's rows; the finished rows of the group before
    if (gi + 1 < ng) request(gi + 1, next);
    if (!STATE_ONLY && gi > 0) store_rows(gi - 1, Ol);

    if (n < C) {                                 // (the last group of all: the powers are not needed again)
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = 16 * ks + 8 * hi + j;
          fv[ks][j] = i < n ? decay_pow(g2, n - 1 - i) : 0.f;
        }
    }
    // (addresses kept over the loop would not fit the registers)
    Swizzled<D> kv = kv0, kx = kx0;
    kv.forget_rows(); kv.forget_cols(); kx.forget_cols();
    int t16 = tile16;
    asm volatile("" : "+v"(t16));
    bf16x8 vop[4];                               // V[16ks + 8hi + 0..7][32 ct + l32]
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) vop[ks] = kv.cols(Vl, 16 * ks, ct);

    f32x16 O;
    if (!STATE_ONLY) {
      // ---- this wave's tiles of P^T, weighted
#pragma unroll
      for (int i = 0; i < G::TW; ++i) {
        const int nt = w + i * G::NW, tb = tile_row(nt), sb = nt - tb * (tb + 1) / 2;
        if (nt < 10) {
          bf16x8 ko[D / 32], qo[D / 32];
#pragma unroll
          for (int ks = 0; ks < D / 32; ++ks) {
            ko[ks] = lds_row8(Kl + 16 * sb * D + (t16 ^ (ks << 3)));
            qo[ks] = lds_row8(Ql + 16 * tb * D + (t16 ^ (ks << 3)));
          }
          __builtin_amdgcn_sched_barrier(0);
          f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < D / 32; ++ks) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ko[ks], qo[ks], x, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) x[r] = fac[i][r] != 0.f ? x[r] * fac[i][r] : 0.f;
          *reinterpret_cast<u32x2*>(Pl + Swizzled<C>::piece(16 * tb + l16, 2 * sb + (q4 >> 1)) + 4 * (q4 & 1)) =
              u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);           // (the rest's reads ahead of the scores would cost registers)
    // (what a step's products read is asked for during the step before, the scores' all at once: 273 -> 264 us)
    bf16x8 qn[4], qa[4], kc[4][G::IT];
    auto read = [&](int ks) {
      if (ks > 3) return;
      if (!STATE_ONLY && ks < 2 * G::IT) {
        qn[ks] = kv.rows(Ql, 32 * half, 2 * G::IT * half + ks);
        qa[ks] = kv.rows(Ql, 32 * (1 - half), 2 * G::IT * half + ks);
      }
#pragma unroll
      for (int it = 0; it < G::IT; ++it) kc[ks][it] = kx.cols(Kl, 16 * ks, G::IT * half + it);
    };
    read(0);
    // ---- S^T Q^T over this wave's rows of S: its own queries' and, for the other wave of the pair, that one's
    bf16x8 sop[2 * G::IT];
    if (!STATE_ONLY) {
#pragma unroll
      for (int i = 0; i < 2 * G::IT; ++i) sop[i] = pack8(S[i / 2], 8 * (i % 2));
    }
    // ---- the state takes the group
    // (a branch of the whole workgroup: a select in every element costs twice as much, 2.7 % of the long prompts)
    if (n < C) {
      const Fade fade(a.log_decay, h, n);
#pragma unroll
      for (int it = 0; it < G::IT; ++it)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[it][r] = fade.of(S[it][r]);
    } else if (slow64) {
#pragma unroll
      for (int it = 0; it < G::IT; ++it) S[it] += S[it] * fade64.f;
    } else {
#pragma unroll
      for (int it = 0; it < G::IT; ++it) S[it] *= fade64.f;
    }
    f32x16 away = {};
    O = f32x16{};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      __builtin_amdgcn_sched_barrier(0);
      read(ks + 1);
      if (!STATE_ONLY && ks < 2 * G::IT) {
        O = mfma(sop[ks], qn[ks], O);
        away = mfma(sop[ks], qa[ks], away);
      }
      f32x16 x;                                  // eight values; split8 takes them from an accumulator
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (float)vop[ks][j] * fv[ks][j];
      bf16x8 vt[3];
      split8(x, 0, vt[0], vt[1]);
      if (TERMS == 3) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] - (float)vt[0][j] - (float)vt[1][j];
        vt[2] = pack8(x, 0);
      }
#pragma unroll
      for (int i = 0; i < TERMS; ++i)
#pragma unroll
        for (int it = 0; it < G::IT; ++it) S[it] = mfma(kc[ks][it], vt[i], S[it]);
    }
    if (!STATE_ONLY) {
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<f32x4*>(Xl + (w * 4 + r4) * 256 + 4 * lane) = f32x4{away[4 * r4], away[4 * r4 + 1], away[4 * r4 + 2], away[4 * r4 + 3]};
    }
    if (!STATE_ONLY) {
      __syncthreads();                           // P; the read-outs from the other half's rows
      const float* X = Xl + ((w + G::CT) % G::NW * 4) * 256 + 4 * lane;
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 y = *reinterpret_cast<const f32x4*>(X + r4 * 256);
#pragma unroll
        for (int i = 0; i < 4; ++i) O[4 * r4 + i] = (O[4 * r4 + i] + y[i]) * fq;
      }
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
        if (ks < 2 || half) O = mfma(vop[ks], pr.rows(Pl, 32 * half, ks), O);
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<u32x2*>(Ol + Swizzled<D>::piece(32 * half + l32, 4 * ct + r4) + 4 * hi) =
            u32x2{pack_bf16x2(O[4 * r4], O[4 * r4 + 1]), pack_bf16x2(O[4 * r4 + 2], O[4 * r4 + 3])};
    }
  };
  for (int gi = 0; gi < ng; gi += 2) {           // (two at a time: the buffers' addresses are constants.  __restrict: see Fetch)
    group(gi, even, odd, Pl, Xl, Ol);
    if (gi + 1 < ng) group(gi + 1, odd, even, Pl, Xl, Ol);
  }
  if (!STATE_ONLY) {
    if (ng > 0) {
      __syncthreads();
      store_rows(ng - 1, Ol);
    }
    // rows behind the end of the sequence, in groups that the walk has not met
    for (int e = tid; e < (t_end - t_begin - ng * C) * G::PPR; e += G::NT) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      *reinterpret_cast<u32x4*>(gout + (int64_t)(t_begin + ng * C + e / G::PPR) * wo.t + e % G::PPR * 8) = z;
    }
  }
  float* So = STATE_ONLY ? slots + (size_t)seg * (D * D) : a.S_out && seg == a.nseg - 1 ? a.S_out + (size_t)bh * D * D : nullptr;
  if (So) {
#pragma unroll
    for (int it = 0; it < G::IT; ++it)
#pragma unroll
      for (int r = 0; r < 16; ++r) So[at(it, r)] = S[it][r];
  }
}

template <int D, bool STATE_ONLY, int TERMS>
hipError_t launch(const DecayArgs& a, hipStream_t s) {
  using G = Cfg<D>;
  constexpr int bytes = STATE_ONLY ? G::KV : G::ALL;
  hipError_t e = LINATTN_MAX_LDS_ONCE((decay_prefill_kernel<D, STATE_ONLY, TERMS>), bytes);
  if (e != hipSuccess) return e;
  decay_prefill_kernel<D, STATE_ONLY, TERMS><<<dim3(a.roles * a.B * a.H * (STATE_ONLY ? (a.nseg - 1) * a.pieces : a.nseg)), G::NT, bytes, s>>>(a);
  return hipGetLastError();
}

template <bool STATE_ONLY>
hipError_t launch_d(const DecayArgs& a, int d, hipStream_t s) {
  if (a.S_out) return d == 64 ? launch<64, STATE_ONLY, 3>(a, s) : launch<128, STATE_ONLY, 3>(a, s);
  return d == 64 ? launch<64, STATE_ONLY, 2>(a, s) : launch<128, STATE_ONLY, 2>(a, s);
}

}  // namespace

hipError_t launch_decay_first_pass_bf16(const DecayArgs& a, int d, hipStream_t s) { return launch_d<true>(a, d, s); }
hipError_t launch_decay_rows_bf16(const DecayArgs& a, int d, hipStream_t s) { return launch_d<false>(a, d, s); }

}  // namespace linattn
