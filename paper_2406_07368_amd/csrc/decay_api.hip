// C ABI of linear attention with a decay (include/linattn.h): argument validation, launch planning, dispatch.
#include "../../include/linattn.h"

#include <hip/hip_runtime.h>

#include "common.h"
#include "decay.h"
#include "rows.h"

using namespace linattn;

namespace {

// The state before every segment from what the segments add to it: S_{s+1} = lambda^{tokens of s} S_s + inc_s.  A thread
// owns one element, so that every request is a whole row; the increments of sixteen segments are requested at a time, the first
// ahead of the factors (6.2 -> 4.7 us at 8 heads of 128 over 1000 tokens).
__global__ __launch_bounds__(256) void decay_scan_kernel(DecayArgs a, int dd) {
  const int per = dd / 256, bhr = blockIdx.x / per, e = blockIdx.x % per * 256 + threadIdx.x;
  const int bh = bhr / a.roles, b = bh / a.H;
  const int len = clamp_len(a.lens, b, a.L);
  float* p = a.ws + (size_t)bhr * a.nseg * dd + e;
  float x = a.S_in ? a.S_in[(size_t)bh * dd + e] : 0.f;
  float inc[16];
  auto request = [&](int s0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) inc[i] = s0 + i < a.nseg - 1 ? p[(size_t)(s0 + i) * dd] : 0.f;
  };
  request(0);
  const Fade whole(a.log_decay, bh % a.H, a.seg_len), end(a.log_decay, bh % a.H, len % a.seg_len);   // (over a segment; over the one that the sequence ends in)
  for (int s0 = 0; s0 < a.nseg; s0 += 16) {
    if (s0 > 0) request(s0);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (s0 + i < a.nseg) {
        p[(size_t)(s0 + i) * dd] = x;
        const int n = segment_tokens(s0 + i, a.seg_len, len);
        x = (n == a.seg_len ? whole.of(x) : n > 0 ? end.of(x) : x) + inc[i];
      }
  }
}

// the state of one head through a call without tokens
__global__ __launch_bounds__(256) void state_through_kernel(const float* from, float* to, int dd) {
  for (int i = threadIdx.x; i < dd; i += 256) to[(size_t)blockIdx.x * dd + i] = from ? from[(size_t)blockIdx.x * dd + i] : 0.f;
}

// Up to so many segments every segment sums up for itself what those before it add (64 KB each at d = 128, from the L2 cache)
// instead of a launch that does.  Where there are two, the first pass has one of them to do, and cuts it into two pieces.
constexpr int kFold = 4;

struct Plan {
  int nseg, seg_len, pieces;
  size_t bytes;
};
// A walk needs a compute unit (bf16 rows of 128: its two row buffers take 120 KB of LDS; fp32: the matrix cores; rows of 64: half of
// one).  Where there are fewer walks the sequence is cut into segments of two groups or more (fp32, whose groups take longer: one), for
// one more read of K and V, if what that saves -- of `groups` steps all but 1/n, and half as many steps of the first pass -- makes up
// for the second launch: some four steps of bf16 (d = 128, 120 walks in two segments: 44 us of 47 at 16 groups, but 30 of 27 at 8),
// half a one of fp32.
// Where more than half of the chip is busy none is cut: segments of more walks than have room run in two rounds (d = 128, bf16, 130 walks
// of 4096 tokens: whole 208 us, in two 286, in three 240; 250 walks: 263, 351, 378; fp32 943, 1169, 947 and 963, 1197, 1291).
Plan plan(const linattn_decay_desc* d, int32_t L, int roles) {
  Plan p{1, L, 1, 0};
  const bool f32 = d->io_dtype == LINATTN_F32;
  const int64_t walks = (int64_t)roles * d->B * d->H, room = d->d == 128 ? 256 : 512;
  const int groups = (L + 63) / 64, least = f32 ? 1 : 2;
  int64_t n = room / walks;
  if (n > groups / least) n = groups / least;
  if (n > 64) n = 64;
  if (2 * groups * n - 3 * groups < (f32 ? 1 : 8) * n) n = 1;
  if (n > 1) {
    p.pieces = n == 2 && groups >= 4 * least ? 2 : 1;
    p.seg_len = (int)((groups + n * p.pieces - 1) / (n * p.pieces)) * 64 * p.pieces;
    p.nseg = (L + p.seg_len - 1) / p.seg_len;
    if (p.nseg > 1) p.bytes = (size_t)walks * p.nseg * p.pieces * d->d * d->d * sizeof(float);
  }
  return p;
}

linattn_status check(const linattn_decay_desc* d, int32_t L, bool gradient, bool strides = true) {
  if (!d) return LINATTN_ERR_NULL;
  if (d->io_dtype != LINATTN_F32 && d->io_dtype != LINATTN_BF16) return LINATTN_ERR_DTYPE;
  if (d->B < 1 || d->H < 1 || (int64_t)d->B * d->H > (int64_t)1 << 20) return LINATTN_ERR_SHAPE;
  if (d->d != 64 && d->d != 128) return LINATTN_ERR_SHAPE;
  if (!finite(d->scale) || d->reserved != 0 || L < 0 || L > kMaxTokens) return LINATTN_ERR_SHAPE;
  if (!strides) return LINATTN_OK;
  bool ok = good_input(d->q, d->B, d->H, L) && good_input(d->k, d->B, d->H, L) && good_input(d->v, d->B, d->H, L);
  if (gradient)
    ok = ok && good_input(d->dout, d->B, d->H, L) && good_output(d->dq, d->B, d->H, L, d->d) && good_output(d->dk, d->B, d->H, L, d->d) &&
         good_output(d->dv, d->B, d->H, L, d->d);
  else
    ok = ok && good_output(d->out, d->B, d->H, L, d->d);
  return ok ? LINATTN_OK : LINATTN_ERR_SHAPE;
}

linattn_status run(DecayArgs& a, const linattn_decay_desc* d, const Plan& p, void* workspace, hipStream_t s) {
  a.B = d->B; a.H = d->H; a.scale = d->scale;
  a.nseg = p.nseg; a.seg_len = p.seg_len; a.pieces = 1; a.piece_len = p.seg_len; a.ws = static_cast<float*>(workspace);
  const bool bf16 = d->io_dtype == LINATTN_BF16;
  hipError_t e = hipSuccess;
  if (p.nseg > 1) {
    // (in place: the last segment writes the state that the others would read)
    a.fold = p.nseg <= kFold && !(a.S_in && a.S_in == a.S_out);
    a.pieces = a.fold ? p.pieces : 1; a.piece_len = p.seg_len / a.pieces;
    e = bf16 ? launch_decay_first_pass_bf16(a, d->d, s) : launch_decay_first_pass_f32(a, d->d, s);
    if (e == hipSuccess && !a.fold) {
      const int dd = d->d * d->d;
      decay_scan_kernel<<<dim3(a.roles * a.B * a.H * (dd / 256)), 256, 0, s>>>(a, dd);
      e = hipGetLastError();
    }
  }
  if (e == hipSuccess) e = bf16 ? launch_decay_rows_bf16(a, d->d, s) : launch_decay_rows_f32(a, d->d, s);
  return e == hipSuccess ? LINATTN_OK : LINATTN_ERR_HIP;
}

}  // namespace

extern "C" {

size_t linattn_decay_workspace_bytes(const linattn_decay_desc* desc, int32_t L) {
  return check(desc, L, false) == LINATTN_OK && L > 0 ? plan(desc, L, 1).bytes : 0;
}
size_t linattn_decay_backward_workspace_bytes(const linattn_decay_desc* desc, int32_t L) {
  return check(desc, L, true) == LINATTN_OK && L > 0 ? plan(desc, L, 3).bytes : 0;
}

linattn_status linattn_decay_prefill(const linattn_decay_desc* desc, int32_t L, const void* q, const void* k, const void* v,
                                     const float* log_decay, const int32_t* lens, const float* S_in, void* out, float* S_out,
                                     void* workspace, size_t workspace_bytes, void* hip_stream) {
  const linattn_status st = check(desc, L, false);
  if (st != LINATTN_OK) return st;
  if (!log_decay || (L > 0 && (!q || !k || !v || !out))) return LINATTN_ERR_NULL;
  if (!aligned16_all({q, k, v, log_decay, lens, S_in, out, S_out, workspace})) return LINATTN_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (L == 0) {                                            // the state through
    if (S_out && S_out != S_in) {
      state_through_kernel<<<dim3(desc->B * desc->H), 256, 0, s>>>(S_in, S_out, desc->d * desc->d);
      if (hipGetLastError() != hipSuccess) return LINATTN_ERR_HIP;
    }
    return LINATTN_OK;
  }
  const Plan p = plan(desc, L, 1);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return LINATTN_ERR_WORKSPACE;
  DecayArgs a{};
  a.role[0] = {rows(q, desc->q), rows(k, desc->k), rows(v, desc->v), rows(out, desc->out), 0};
  a.roles = 1; a.L = L; a.log_decay = log_decay; a.lens = lens; a.S_in = S_in; a.S_out = S_out;
  return run(a, desc, p, workspace, s);
}

linattn_status linattn_decay_backward(const linattn_decay_desc* desc, int32_t L, const void* q, const void* k, const void* v,
                                      const float* log_decay, const int32_t* lens, const void* dout, void* dq, void* dk, void* dv,
                                      void* workspace, size_t workspace_bytes, void* hip_stream) {
  const linattn_status st = check(desc, L, true);
  if (st != LINATTN_OK) return st;
  if (!log_decay || (L > 0 && (!q || !k || !v || !dout || !dq || !dk || !dv))) return LINATTN_ERR_NULL;
  if (!aligned16_all({q, k, v, log_decay, lens, dout, dq, dk, dv, workspace})) return LINATTN_ERR_ALIGN;
  if (L == 0) return LINATTN_OK;
  const Plan p = plan(desc, L, 3);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return LINATTN_ERR_WORKSPACE;
  DecayArgs a{};
  const Rows rq = rows(q, desc->q), rk = rows(k, desc->k), rv = rows(v, desc->v), rd = rows(dout, desc->dout);
  a.role[0] = {rd, rv, rk, rows(dq, desc->dq), 0};
  a.role[1] = {rv, rd, rq, rows(dk, desc->dk), 1};
  a.role[2] = {rk, rq, rd, rows(dv, desc->dv), 1};
  a.roles = 3; a.L = L; a.log_decay = log_decay; a.lens = lens;
  return run(a, desc, p, workspace, static_cast<hipStream_t>(hip_stream));
}

linattn_status linattn_decay_step(const linattn_decay_desc* desc, int32_t kk, const void* q, const void* k, const void* v,
                                  const float* log_decay, float* S, const int32_t* n_commit, void* out, void* hip_stream) {
  const linattn_status st = check(desc, 0, false, false);
  if (st != LINATTN_OK) return st;
  if (kk < 1 || kk > LINATTN_MAX_DRAFT) return LINATTN_ERR_SHAPE;
  if (!q || !k || !v || !log_decay || !S || !out) return LINATTN_ERR_NULL;
  if (!aligned16_all({q, k, v, log_decay, S, n_commit, out})) return LINATTN_ERR_ALIGN;
  DecayStepArgs a{q, k, v, log_decay, S, n_commit, out, desc->B, desc->H, kk, desc->scale};
  return launch_decay_step(a, desc->d, desc->io_dtype == LINATTN_BF16, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? LINATTN_OK : LINATTN_ERR_HIP;
}

}  // extern "C"
