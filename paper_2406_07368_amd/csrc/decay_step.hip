// kk tokens of linear attention with a decay, from a running state (fp32 throughout).  With lambda the head's decay,
//
//   out_j = scale ( lambda^{j+1} q_j^T S + sum_{i<=j} lambda^{j-i} (q_j.k_i) v_i )
//   S'    = lambda^n S + sum_{i<n} lambda^{n-1-i} k_i v_i^T                          n = drafts that are kept (see Fade)
//
// One read and one write of the state (8 d^2 bytes a head) is all the traffic that counts: HBM bounds it.  Every value
// column is independent of the others, so a workgroup takes CB columns of one head: a thread holds R rows of four
// columns of S in registers -- requested before anything else --, every draft's read-out is a sum over a thread's rows,
// the lanes of a wave that share columns, and the four waves; the same registers then take the kept drafts and go back.
// The products of the drafts among themselves (at most 136) are made by every workgroup of a head again: they cost
// less than a launch of their own or a wider workgroup's wait.  Measured: four drafts on 1024 heads of 128 26 us, 5.3 TB/s (32
// columns a workgroup: a 128-byte line per row; 4096 workgroups of 16 KB).
#include "common.h"
#include "decay.h"

namespace linattn {

namespace {

// (eight waves on a SIMD, where LDS has room for them: left alone the compiler takes registers for five, 27.5 -> 27.8 us)
template <typename IO, int D, int CB, int KK>
__global__ __launch_bounds__(256, KK <= 8 ? 8 : 5) void decay_step_kernel(DecayStepArgs a) {
  constexpr int LG = CB / 4;              // lanes side by side on a row's columns
  constexpr int NG = 256 / LG;            // row groups
  constexpr int R = D / NG;               // rows of S per thread
  constexpr int NB = D / CB;
  static_assert(R >= 1 && (LG == 8 || LG == 16), "");
  __shared__ float ql[KK][D], kl[KK][D];
  __shared__ __attribute__((aligned(16))) float vl[KK][CB];
  __shared__ float al[KK][KK];
  __shared__ __attribute__((aligned(16))) float red[4][KK][CB];
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  const int bh = blockIdx.x / NB, c0 = blockIdx.x % NB * CB;
  const int h = bh % a.H, b = bh / a.H, kk = a.kk;
  const int c = 4 * (tid % LG), g = tid / LG;
  float* S = a.S + (size_t)bh * D * D + c0 + c;
  f32x4 s[R];
#pragma unroll
  for (int r = 0; r < R; ++r) s[r] = *reinterpret_cast<const f32x4*>(S + (size_t)(g + NG * r) * D);
  const size_t row0 = (size_t)bh * kk * D;
  for (int e = tid; e < KK * D; e += 256) {
    const bool in = e < kk * D;
    (&ql[0][0])[e] = in ? IO::load1(a.q, row0 + e) : 0.f;
    (&kl[0][0])[e] = in ? IO::load1(a.k, row0 + e) : 0.f;
  }
  for (int e = tid; e < KK * CB; e += 256) {
    const int j = e / CB;
    vl[j][e % CB] = j < kk ? IO::load1(a.v, row0 + (size_t)j * D + c0 + e % CB) : 0.f;
  }
  const float g2 = decay_log2(a.log_decay, h);
  int n = kk;
  if (a.n_commit) {
    n = a.n_commit[b];
    n = n < 0 ? 0 : n > kk ? kk : n;
  }
  const Fade fade(a.log_decay, h, n);
  __syncthreads();
  // q_j . k_i, eight lanes each
  for (int p = tid >> 3; p < KK * KK; p += 32) {
    const int j = p / KK, i = p % KK;
    float x = 0.f;
    if (i <= j) {
      for (int f = tid & 7; f < D; f += 8) x += ql[j][f] * kl[i][f];
    }
    x = sum_lanes<8>(x);
    if ((tid & 7) == 0) al[j][i] = i <= j ? x * decay_pow(g2, j - i) : 0.f;
  }
  // q_j^T S over this thread's rows, the wave's, the workgroup's
#pragma unroll
  for (int j = 0; j < KK; ++j) {
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < R; ++r) x += ql[j][g + NG * r] * s[r];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y = x[i];
      if (LG == 8) y = add_xor8(y);
      y = add_xor16(y);
      x[i] = add_xor32(y);
    }
    if (lane < LG) *reinterpret_cast<f32x4*>(&red[w][j][c]) = x;
  }
  __syncthreads();
  for (int e = tid; e < KK * CB; e += 256) {
    const int j = e / CB, cc = e % CB;
    if (j < kk) {
      float x = (red[0][j][cc] + red[1][j][cc] + red[2][j][cc] + red[3][j][cc]) * decay_pow(g2, j + 1);
      for (int i = 0; i <= j; ++i) x += al[j][i] * vl[i][cc];
      IO::store1(a.out, row0 + (size_t)j * D + c0 + cc, x * a.scale);
    }
  }
  if (n == 0) return;
  // what the state loses and gains goes into it in one rounding (a loss of less than 2^-25 of it would be lost alone)
  f32x4 more[R];
#pragma unroll
  for (int r = 0; r < R; ++r) more[r] = s[r] * fade.f;
  for (int i = 0; i < n; ++i) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(&vl[i][c]) * decay_pow(g2, n - 1 - i);
#pragma unroll
    for (int r = 0; r < R; ++r) more[r] += kl[i][g + NG * r] * x;
  }
#pragma unroll
  for (int r = 0; r < R; ++r) s[r] = fade.slow ? s[r] + more[r] : more[r];
#pragma unroll
  for (int r = 0; r < R; ++r) *reinterpret_cast<f32x4*>(S + (size_t)(g + NG * r) * D) = s[r];
}

template <typename IO, int D, int CB>
void launch(const DecayStepArgs& a, hipStream_t s) {
  const dim3 grid(a.B * a.H * (D / CB));
  if (a.kk == 1) decay_step_kernel<IO, D, CB, 1><<<grid, 256, 0, s>>>(a);
  else if (a.kk == 2) decay_step_kernel<IO, D, CB, 2><<<grid, 256, 0, s>>>(a);
  else if (a.kk <= 4) decay_step_kernel<IO, D, CB, 4><<<grid, 256, 0, s>>>(a);
  else if (a.kk <= 8) decay_step_kernel<IO, D, CB, 8><<<grid, 256, 0, s>>>(a);
  else decay_step_kernel<IO, D, CB, 16><<<grid, 256, 0, s>>>(a);
}

template <typename IO>
void launch_d(const DecayStepArgs& a, int d, hipStream_t s) {
  if (d == 64) launch<IO, 64, 32>(a, s);
  else launch<IO, 128, 32>(a, s);
}

}  // namespace

hipError_t launch_decay_step(const DecayStepArgs& a, int d, bool bf16, hipStream_t s) {
  if (bf16) launch_d<IoBf16>(a, d, s);
  else launch_d<IoF32>(a, d, s);
  return hipGetLastError();
}

}  // namespace linattn
