// Linear attention with a decay for each head: launch interfaces between the C-ABI layer (decay_api.hip) and the
// kernels, and what the kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace linattn {

struct Rows {              // rows [B,H,L,d] of a tensor, addressed by element strides
  const void* p;
  int64_t b, h, t;
};

// out_t = scale sum_{s<=t} lambda^{t-s} (q_t . k_s) v_s, or with `reverse` the same over s >= t.  The gradient is three
// of these with the roles of the tensors changed, so a launch carries up to three.
struct DecayRole {
  Rows q, k, v, out;
  int reverse;
};
struct DecayArgs {
  DecayRole role[3];
  int roles;
  const float* log_decay;  // [H]
  const int32_t* lens;     // [B] or null
  const float* S_in;       // [B,H,d,d] or null (one role only)
  float* S_out;            // or null
  float* ws;               // nseg > 1: [B*H][roles][nseg * pieces][d*d], the state before every segment, or, with fold, what every piece adds
  int B, H, L;
  int nseg, seg_len;       // segments of seg_len tokens (a multiple of 64), in the order of the walk
  int fold;                // few segments: each sums up what those before it add
  int pieces, piece_len;   // of a segment in the first pass (1 without fold)
  float scale;
};
hipError_t launch_decay_first_pass_bf16(const DecayArgs& a, int d, hipStream_t s);
hipError_t launch_decay_rows_bf16(const DecayArgs& a, int d, hipStream_t s);
hipError_t launch_decay_first_pass_f32(const DecayArgs& a, int d, hipStream_t s);
hipError_t launch_decay_rows_f32(const DecayArgs& a, int d, hipStream_t s);

struct DecayStepArgs {
  const void *q, *k, *v;   // [B,H,kk,d] dense
  const float* log_decay;
  float* S;                // [B,H,d,d] in/out
  const int32_t* n_commit;
  void* out;
  int B, H, kk;
  float scale;
};
hipError_t launch_decay_step(const DecayStepArgs& a, int d, bool bf16, hipStream_t s);

// log2 lambda of a head: log_decay <= 0, what is above 0 and NaN read as 0.  The lower bound keeps the products with a
// count of tokens finite (and 0 * it at 0, where -inf would give NaN); 2 to any of them but 0 is 0 all the same.
__device__ __forceinline__ float decay_log2(const float* log_decay, int h) {
  const float g = log_decay[h] * 1.44269504088896340736f;
  return g < 0.f ? fmaxf(g, -1e30f) : 0.f;
}
// What a running state x becomes over n >= 0 tokens: slow ? x + x f : x f.  A factor near 1 held as such is off by up to 2^-24, always
// to the same side, and a state that lives through thousands of steps of a slow head meets it in every one of them: lambda^n - 1 has
// all its bits.  Where lambda^n is 1/2 or less the difference would cancel, and what is left of the state is right by its factor.
struct Fade {
  float f;
  bool slow;
  __device__ __forceinline__ Fade(const float* log_decay, int h, int n) {
    const float g = log_decay[h], less = g < 0.f ? expm1f(fmaxf(g, -1e30f) * (float)n) : 0.f;
    slow = less > -0.5f;
    f = slow ? less : __builtin_amdgcn_exp2f(decay_log2(log_decay, h) * (float)n);
  }
  __device__ __forceinline__ float of(float x) const { return slow ? x + x * f : x * f; }
};
// lambda^n, n >= 0
__device__ __forceinline__ float decay_pow(float g2, int n) { return __builtin_amdgcn_exp2f(g2 * (float)n); }

// Which row the walk's step i is: behind the end of a sequence the rows in their own order (they are only zeroed).
__device__ __forceinline__ int walk_row(int i, int len, int reverse) { return reverse && i < len ? len - 1 - i : i; }
__device__ __forceinline__ int clamp_len(const int32_t* lens, int b, int L) {
  if (!lens) return L;
  const int n = lens[b];
  return n < 0 ? 0 : n > L ? L : n;
}

// tokens of segment j of a sequence of len
__device__ __forceinline__ int segment_tokens(int j, int seg_len, int len) {
  const int left = len - j * seg_len;
  return left < 0 ? 0 : left > seg_len ? seg_len : left;
}

}  // namespace linattn
