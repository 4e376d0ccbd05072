// Softmax attention over a sliding window with sinks: launch interfaces between the C-ABI layer (window_api.hip) and
// the kernels, and what the kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "decay.h"   // Rows, clamp_len
#include "swizzle.h"

namespace linattn {

struct WindowArgs {
  Rows q, k, v, out;
  Rows dout, dq, dk, dv;          // gradient
  const int32_t* lens;
  float* lse;                     // [B,H,L]: written by the prefill (may be null), read by the gradient
  float* stats;                   // gradient: [2][B,H,L], lse in base 2 and dout . out
  int far;                        // gradient: workgroups per key/value head for the queries that see only sinks of key tile 0
  int parts;                      // gradient: workgroups per key tile
  float* sink_part;               // far > 0: [B*H_kv][parts + 2 far][2][sinks][d], shares of the sinks' dk, dv
  float* part;                    // parts > 1: [B*H_kv][parts][2][L][d], shares of the other rows'
  int B, H, Hkv, L;
  int window, sinks;
  float scale;
  float dk_scale;                 // gradient: scale, or 0 where every token sees only itself
};
hipError_t launch_window_prefill_bf16(const WindowArgs& a, int d, hipStream_t s);
hipError_t launch_window_prefill_f32(const WindowArgs& a, int d, hipStream_t s);
hipError_t launch_window_backward(const WindowArgs& a, int d, hipStream_t s);

constexpr int kWindowQ = 32, kWindowKeys = 128;   // gradient of k and v: queries at a time, keys of a workgroup
// the first tile of kWindowQ queries that sees nothing of key tile 0 but its sinks
__host__ __device__ inline int window_far_tile(int64_t window) {
  const int64_t t = (kWindowKeys - 1 + window - 1) / kWindowQ + 1;
  return t > 0x7fffffff ? 0x7fffffff : (int)t;
}

struct WindowStepArgs {
  const void *q, *k, *v;          // [B,H,kk,d], [B,Hkv,kk,d] dense
  void *kcache, *vcache;          // [B,Hkv,sinks+window,d]
  int32_t* pos;                   // [B,Hkv]
  const int32_t* n_commit;
  void* out;
  float* ws;                      // nsplit > 1: [B*Hkv][nsplit][R][d] sums, then [B*Hkv][nsplit][R][2] maximum and weight
  int B, H, Hkv, kk;
  int window, sinks, nsplit;
  float scale;
};
int window_step_splits(int64_t heads, int64_t held, int rows);
hipError_t launch_window_step(const WindowStepArgs& a, int d, bool bf16, hipStream_t s);

struct WindowCacheArgs {
  Rows k, v;
  const int32_t* lens;
  void *kcache, *vcache;
  int32_t* pos;
  int B, Hkv, L, window, sinks;
};
hipError_t launch_window_cache(const WindowCacheArgs& a, int d, bool bf16, hipStream_t s);

// exponents in base 2; a scale of 0 becomes one that leaves the scores equal (0 * -inf would not)
__device__ __forceinline__ float window_log2_scale(float scale) { return fmaxf(scale * 1.44269504088896340736f, 1e-30f); }

// Token t sees token s.  (window >= 1, both below 2^31: t - window does not overflow)
__device__ __forceinline__ bool window_sees(int t, int s, int window, int sinks) { return s <= t && (s > t - window || s < sinks); }

// The accumulator of a 32 x 32 product: which row register r of a lane of half `hi` holds.
__device__ __forceinline__ int acc_row(int r, int hi) { return (r & 3) + 8 * (r >> 2) + 4 * hi; }

// max(x[l], x[l ^ 32])
__device__ __forceinline__ float max_xor32(float x) {
  const unsigned u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Consecutive workgroups go to the eight chiplets in turn, each with an L2 of its own.  The `units` (a key/value head of a
// batch row) of `each` workgroups, which read the same keys, are dealt out whole where every chiplet gets (nearly) as many;
// else a chiplet takes a run of neighbours.  A launch has xcd_grid workgroups; a place >= units * each has no work.
__host__ __device__ inline bool xcd_whole(int units) { return units % 8 == 0 || units >= 64; }
__host__ __device__ inline int64_t xcd_grid(int units, int each) {
  return xcd_whole(units) ? (int64_t)((units + 7) / 8) * 8 * each : ((int64_t)units * each + 7) / 8 * 8;
}
__device__ __forceinline__ int xcd_place(int block, int units, int each) {
  const int x = block % 8, i = block / 8;
  if (!xcd_whole(units)) return x * ((units * each + 7) / 8) + i;
  const int u = x + 8 * (i / each);
  return u < units ? u * each + i % each : units * each;
}

}  // namespace linattn
