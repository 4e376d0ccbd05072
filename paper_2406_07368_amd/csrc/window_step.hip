// Steps of softmax attention over a sliding window with sinks: kk tokens behind a cache of rows.
//
// The cache of a key/value head holds token s < sinks in row s and any other in row sinks + (s - sinks) % window, so at
// most sinks + window rows however long the sequence.  With `pos` tokens seen, ring row r holds the token of age
// (pos - sinks - 1 - r) mod window (0 = the newest), if that many went into the ring; token pos + j sees ages below
// window - 1 - j, the sinks, and the step's own tokens up to itself.
//
// The cache is read once whatever the number of query heads that share it and of tokens: their R = (H / H_kv) kk rows are
// the 32 columns of one product (32 at a time).  Tiles of 32 rows -- the step's own tokens are tile 0 -- go round over the
// waves of the workgroups of a head, each with a running maximum and sum of its own and no barrier on the way: S^T = K Q^T
// with the keys straight from memory as the operand, then O^T += V^T P^T with the weights as they stand (bf16 rows of V
// through a wave's own LDS for the transposed reads; fp32 rows straight from memory, on the fp32 matrix instructions).  For bf16
// rows a weight enters as the sum of two bf16 terms, sixteen significant bits: the error of the outputs is that of their own
// rounding (1.67e-3 in the 2-norm; with one term 2.28e-3), for 2 % of the time at the size below (90 -> 92 us).
// The waves' sums are joined in LDS, the workgroups' by a second launch, which also moves the kept tokens into the cache;
// where a head has one workgroup, that does it itself.
//
// Bound: HBM (4 d bytes of cache row a token and key/value head in bf16).  Measured at 256 heads of 128 with windows of up to 4096: 105 us,
// 4.1 TB/s; 8 heads with a window of 2048: 15 us, two launches.
#include "common.h"
#include "kernels.h"
#include "mfma_util.h"
#include "window.h"

namespace linattn {

namespace {

constexpr int KT = 32;
constexpr float kLate = 8.f;                     // log2: how far a running maximum may lie behind before the sums are scaled anew
constexpr float kNone = -1e30f;                  // the maximum over nothing: finite, so that differences are numbers

template <int D>
struct MatBf16 {
  typedef uint16_t elem;
  typedef IoBf16 io;
  static constexpr int LDS = KT * D * 2;         // bytes per wave
  static constexpr int WAVES = 2;                // per SIMD
  static constexpr int PPR = D / 8;
  bf16x8 q[D / 16], k[D / 16];
  u32x4 v[D / 16];
  __device__ __forceinline__ void load_q(const elem* row, int hi) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) q[i] = *reinterpret_cast<const bf16x8*>(row + 16 * i + 8 * hi);
  }
  // key row lane % 32 and the value rows of a tile; those from `rows` on are not there (they re-read its row 0)
  __device__ __forceinline__ void request_k(const elem* kb, int rows, int lane) {
    const elem* kr = kb + ((lane & 31) < rows ? lane & 31 : 0) * D + 8 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) k[i] = *reinterpret_cast<const bf16x8*>(kr + 16 * i);
  }
  __device__ __forceinline__ void request_v(const elem* vb, int rows, int lane) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const int p = lane + 64 * i, r = p / PPR;
      v[i] = *reinterpret_cast<const u32x4*>(vb + (r < rows ? r : 0) * D + p % PPR * 8);
    }
  }
  // the value rows -> the wave's LDS, from where add() takes them; its registers are free for the next tile's
  static constexpr bool STAGED = true;
  __device__ __forceinline__ void stage(unsigned char* lds, int rows, int lane) {
    uint16_t* Vl = reinterpret_cast<uint16_t*>(lds);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const int e = lane + 64 * i;
      *reinterpret_cast<u32x4*>(Vl + Swizzled<D>::piece(e / PPR, e % PPR)) = e / PPR < rows ? v[i] : u32x4{0u, 0u, 0u, 0u};
    }
    __builtin_amdgcn_wave_barrier();             // (one wave: its LDS operations are served in order)
  }
  __device__ __forceinline__ f32x16 scores() const {
    f32x16 x = {};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) x = mfma(k[i], q[i], x);
    return x;
  }
  __device__ __forceinline__ void add(f32x16 (&O)[D / 32], const f32x16& p, const unsigned char* lds, int, int lane) {
    const uint16_t* Vl = reinterpret_cast<const uint16_t*>(lds);
    const Swizzled<D> at(lane, 4);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      bf16x8 w, rest, vt[D / 32];
      split8(p, 8 * half, w, rest);
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct) {
        vt[ct] = at.cols_acc(Vl, 16 * half, ct);
        O[ct] = mfma(vt[ct], w, O[ct]);
      }
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct) O[ct] = mfma(vt[ct], rest, O[ct]);
    }
    __builtin_amdgcn_wave_barrier();
  }
};

template <int D>
struct MatF32 {
  typedef float elem;
  typedef IoF32 io;
  static constexpr int LDS = 0;
  static constexpr int WAVES = 1;
  static constexpr bool STAGED = false;
  f32x4 q[D / 8], k[D / 8];
  float v[16][D / 32];
  __device__ __forceinline__ void load_q(const elem* row, int hi) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) q[i] = *reinterpret_cast<const f32x4*>(row + D / 2 * hi + 4 * i);
  }
  __device__ __forceinline__ void request_k(const elem* kb, int rows, int lane) {
    const elem* kr = kb + ((lane & 31) < rows ? lane & 31 : 0) * D + D / 2 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) k[i] = *reinterpret_cast<const f32x4*>(kr + 4 * i);
  }
  __device__ __forceinline__ void request_v(const elem* vb, int rows, int lane) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = acc_row(r, lane >> 5);
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct) v[r][ct] = vb[(row < rows ? row : 0) * D + 32 * ct + (lane & 31)];
    }
  }
  __device__ __forceinline__ void stage(unsigned char*, int, int) {}
  __device__ __forceinline__ f32x16 scores() const {
    f32x16 x = {};
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i][e], q[i][e], x, 0, 0, 0);
    return x;
  }
  __device__ __forceinline__ void add(f32x16 (&O)[D / 32], const f32x16& p, const unsigned char*, int rows, int lane) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const bool in = acc_row(r, lane >> 5) < rows;
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct) O[ct] = __builtin_amdgcn_mfma_f32_32x32x2f32(in ? v[r][ct] : 0.f, p[r], O[ct], 0, 0, 0);
    }
  }
};

__device__ __forceinline__ int kept(const int32_t* n_commit, int b, int kk) {
  if (!n_commit) return kk;
  const int n = n_commit[b];
  return n < 0 ? 0 : n > kk ? kk : n;
}

// the first n of the step's tokens -> the cache (a token that a later one of them replaces is left out)
template <typename E, int D>
__device__ void commit(const WindowStepArgs& a, int bk, int pos, int n, int tid) {
  constexpr int PPR = D * sizeof(E) / 16, EP = 16 / sizeof(E);
  const int64_t held = (int64_t)a.sinks + a.window;
  for (int e = tid; e < 2 * n * PPR; e += 256) {
    const int kv = e / (n * PPR), j = e / PPR % n, c = e % PPR * EP;
    const int64_t at = (int64_t)pos + j;
    if (at >= a.sinks && at + a.window < (int64_t)pos + n) continue;
    const int64_t row = at < a.sinks ? at : a.sinks + (at - a.sinks) % a.window;
    const E* from = static_cast<const E*>(kv ? a.v : a.k) + ((int64_t)bk * a.kk + j) * D + c;
    E* to = static_cast<E*>(kv ? a.vcache : a.kcache) + (bk * held + row) * D + c;
    *reinterpret_cast<u32x4*>(to) = *reinterpret_cast<const u32x4*>(from);
  }
  if (tid == 0) a.pos[bk] = pos + n;
}

template <template <int> class M, int D>
__global__ __launch_bounds__(256, M<D>::WAVES) void window_step_kernel(WindowStepArgs a) {
  typedef typename M<D>::elem E;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_b[];
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int split = blockIdx.x % a.nsplit, bk = blockIdx.x / a.nsplit;
  const int b = bk / a.Hkv, hk = bk % a.Hkv, group = a.H / a.Hkv, R = group * a.kk;
  const int r0 = 32 * blockIdx.y, row = r0 + l32;    // this lane's query row: head row / kk of the group, token row % kk
  const int j = row % a.kk;
  const int64_t held = (int64_t)a.sinks + a.window;
  const E* kc = static_cast<const E*>(a.kcache) + bk * held * D;
  const E* vc = static_cast<const E*>(a.vcache) + bk * held * D;
  const E* kn = static_cast<const E*>(a.k) + (int64_t)bk * a.kk * D;
  const E* vn = static_cast<const E*>(a.v) + (int64_t)bk * a.kk * D;
  const int64_t qrow = ((int64_t)b * a.H + hk * group) * a.kk;
  const float c = window_log2_scale(a.scale);
  unsigned char* lds = smem_b + w * M<D>::LDS;
  M<D> mat;
  // Tile i's rows: the step's own, or those of the cache from row (i - 1) KT on.  They are requested before it is known how many
  // of them are in use (what is not is dropped later): `pos` costs a trip to memory of its own.
  auto place = [&](int i, const E*& kb, const E*& vb) -> int {
    if (i == 0) { kb = kn; vb = vn; return a.kk; }
    const int64_t s0 = (int64_t)(i - 1) * KT;
    kb = kc + s0 * D; vb = vc + s0 * D;
    return held - s0 < KT ? (int)(held - s0) : KT;
  };
  const int first = split * 4 + w, stride = a.nsplit * 4;
  const E *kb, *vb;
  if (first == 0 || (int64_t)(first - 1) * KT < held) {
    const int n = place(first, kb, vb);
    mat.request_k(kb, n, lane);
    mat.request_v(vb, n, lane);
  }
  mat.load_q(static_cast<const E*>(a.q) + (qrow + (row < R ? row : R - 1)) * D, hi);
  int pos = a.pos[bk];
  pos = pos < 0 ? 0 : pos;
  const int live = pos < held ? pos : (int)held;     // cache rows in use
  const int nt = (live + KT - 1) / KT + 1;
  f32x16 O[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) O[i] = f32x16{};
  float m = kNone, l = 0.f;
  const int ring = pos - a.sinks;                    // tokens that went into the ring (or less than 0)
  for (int i = first; i < nt; i += stride) {
    const int s0 = (i - 1) * KT;                     // the tile's first cache row
    const int rows = i == 0 ? a.kk : live - s0 < KT ? live - s0 : KT;
    const bool more = i + stride < nt;
    int n = 0;
    if (more) n = place(i + stride, kb, vb);
    mat.stage(lds, rows, lane);
    if (M<D>::STAGED && more) mat.request_v(vb, n, lane);
    f32x16 x = mat.scores();
    if (more) mat.request_k(kb, n, lane);
    if (i == 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int s = acc_row(r, hi);
        if (!(s <= j && (s > j - a.window || pos + s < a.sinks))) x[r] = -__builtin_inff();
      }
    } else {
      // age of the tile's first row if it is a ring row; the next rows' are smaller by one each, round the ring
      int age0 = (ring - 1 - (s0 - a.sinks)) % a.window;
      if (age0 < 0) age0 += a.window;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int u = acc_row(r, hi);
        int age = age0 - u;
        if (age < 0) age += a.window;
        if (a.window < KT && age < 0) age = (age0 - u) % a.window + ((age0 - u) % a.window < 0 ? a.window : 0);
        const bool sees = s0 + u < a.sinks ? s0 + u < pos : age < ring && age < a.window - 1 - j;
        if (!sees || u >= rows) x[r] = -__builtin_inff();
      }
    }
    float top = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, x[r]);
    top = max_xor32(top) * c;
    if (__any(top > m + kLate)) {
      const float m2 = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      l *= f;
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct) O[ct] *= f;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r] = __builtin_amdgcn_exp2f(x[r] * c - m);
      l += x[r];
    }
    mat.add(O, x, lds, rows, lane);
    if (!M<D>::STAGED && more) mat.request_v(vb, n, lane);
  }
  l = add_xor32(l);

  // the waves' sums: 2, 3 into 0, 1, then 1 into 0
  float* jl = reinterpret_cast<float*>(smem_b);
#pragma unroll
  for (int half = 2; half >= 1; half /= 2) {
    __syncthreads();
    if (w >= half && w < 2 * half) {
      float* p = jl + (w - half) * (D / 2 + 2) * 64 + lane;
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
        for (int r = 0; r < 16; ++r) p[(16 * ct + r) * 64] = O[ct][r];
      p[D / 2 * 64] = m;
      p[(D / 2 + 1) * 64] = l;
    }
    __syncthreads();
    if (w < half) {
      const float* p = jl + w * (D / 2 + 2) * 64 + lane;
      const float mo = p[D / 2 * 64], m2 = fmaxf(m, mo);
      const float f = __builtin_amdgcn_exp2f(m - m2), fo = __builtin_amdgcn_exp2f(mo - m2);
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[ct][r] = O[ct][r] * f + p[(16 * ct + r) * 64] * fo;
      l = l * f + p[(D / 2 + 1) * 64] * fo;
      m = m2;
    }
  }
  if (w == 0 && row < R) {
    if (a.nsplit == 1) {
      const float inv = 1.f / l;
      E* o = static_cast<E*>(a.out) + (qrow + row) * D;
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const int e = 32 * ct + 8 * r4 + 4 * hi;
          const float y[4] = {O[ct][4 * r4] * inv, O[ct][4 * r4 + 1] * inv, O[ct][4 * r4 + 2] * inv, O[ct][4 * r4 + 3] * inv};
          if constexpr (sizeof(E) == 2) *reinterpret_cast<u32x2*>(o + e) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
          else *reinterpret_cast<f32x4*>(o + e) = f32x4{y[0], y[1], y[2], y[3]};
        }
    } else {
      const int64_t at = ((int64_t)bk * a.nsplit + split) * R + row;
      float* stat = a.ws + (int64_t)a.B * a.Hkv * a.nsplit * R * D + 2 * at;
      if (hi == 0) { stat[0] = m; stat[1] = l; }
      float* o = a.ws + at * D;
      if (l != 0.f) {                                // (0: a share of nothing.  NaN is one of something)
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4)
            *reinterpret_cast<f32x4*>(o + 32 * ct + 8 * r4 + 4 * hi) = f32x4{O[ct][4 * r4], O[ct][4 * r4 + 1], O[ct][4 * r4 + 2], O[ct][4 * r4 + 3]};
      }
    }
  }
  // (every wave is behind the barriers above, so every read of the cache and of pos is done)
  if (a.nsplit == 1 && gridDim.y == 1) commit<E, D>(a, bk, pos, kept(a.n_commit, b, a.kk), tid);
}

// the workgroups' sums; workgroup 0 of a head then moves the kept tokens into the cache
template <typename IO, int D>
__global__ __launch_bounds__(256) void window_join_kernel(WindowStepArgs a) {
  typedef typename IO::elem E;
  constexpr int LR = D / 4, ROWS = 256 / LR;         // threads of a row, rows of a workgroup
  __shared__ float weight[ROWS][64];
  const int bk = blockIdx.x, b = bk / a.Hkv, hk = bk % a.Hkv, group = a.H / a.Hkv, R = group * a.kk;
  const int64_t qrow = ((int64_t)b * a.H + hk * group) * a.kk;
  if (a.nsplit > 1) {
    const int u = threadIdx.x / LR, e = threadIdx.x % LR, row = blockIdx.y * ROWS + u;
    const int64_t at = (int64_t)bk * a.nsplit * R + (row < R ? row : R - 1);
    const float* stat = a.ws + (int64_t)a.B * a.Hkv * a.nsplit * R * D + 2 * at;
    // a thread's shares of the row (at most 64, LR of them at a time), the row's maximum and sum over its threads
    constexpr int EACH = 64 / LR;
    f32x2 st[EACH];
    float m = kNone;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int s = e + LR * i;
      st[i] = s < a.nsplit ? *reinterpret_cast<const f32x2*>(stat + 2 * (int64_t)s * R) : f32x2{kNone, 0.f};
      m = fmaxf(m, st[i][0]);
    }
#pragma unroll
    for (int d = 1; d < LR; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      st[i][0] = __builtin_amdgcn_exp2f(st[i][0] - m);
      l += st[i][1] * st[i][0];
    }
#pragma unroll
    for (int d = 1; d < LR; d *= 2) l += __shfl_xor(l, d);
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < EACH; ++i) weight[u][e + LR * i] = st[i][1] != 0.f ? st[i][0] * inv : -1.f;   // (-1: a share of nothing, which was not written)
    __syncthreads();
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < a.nsplit; ++s) {
      const float f = weight[u][s];                  // (a weight that is NaN, or 0 for values that are, goes into the sum)
      const f32x4 y = *reinterpret_cast<const f32x4*>(a.ws + (at + (int64_t)s * R) * D + 4 * e);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] += f < 0.f ? 0.f : f * y[i];
    }
    if (row < R) {
      E* o = static_cast<E*>(a.out) + (qrow + row) * D + 4 * e;
      if constexpr (sizeof(E) == 2) *reinterpret_cast<u32x2*>(o) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
      else *reinterpret_cast<f32x4*>(o) = x;
    }
  }
  if (blockIdx.y == 0) {
    const int pos = a.pos[bk];
    __syncthreads();
    commit<E, D>(a, bk, pos < 0 ? 0 : pos, kept(a.n_commit, b, a.kk), threadIdx.x);
  }
}

template <template <int> class M, int D>
hipError_t launch(const WindowStepArgs& a, hipStream_t s) {
  typedef typename M<D>::io IO;
  constexpr int JOIN = 2 * (D / 2 + 2) * 64 * 4, LDS = 4 * M<D>::LDS > JOIN ? 4 * M<D>::LDS : JOIN;
  const int R = a.H / a.Hkv * a.kk, blocks = (R + 31) / 32;
  hipError_t e = LINATTN_MAX_LDS_ONCE((window_step_kernel<M, D>), LDS);
  if (e != hipSuccess) return e;
  window_step_kernel<M, D><<<dim3(a.B * a.Hkv * a.nsplit, blocks), 256, LDS, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || (a.nsplit == 1 && blocks == 1)) return e;
  window_join_kernel<IO, D><<<dim3(a.B * a.Hkv, a.nsplit > 1 ? (R * (D / 4) + 255) / 256 : 1), 256, 0, s>>>(a);
  return hipGetLastError();
}

// ---- a prompt's last rows into the cache ---------------------------------------------------------------------------
template <typename E, int D>
__global__ __launch_bounds__(256) void window_cache_kernel(WindowCacheArgs a) {
  constexpr int PPR = D * sizeof(E) / 16, EP = 16 / sizeof(E), PER = 256 / PPR;
  const int bk = blockIdx.x, b = bk / a.Hkv, hk = bk % a.Hkv;
  const int pos = clamp_len(a.lens, b, a.L);
  const int64_t held = (int64_t)a.sinks + a.window;
  const E* k = static_cast<const E*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const E* v = static_cast<const E*>(a.v.p) + b * a.v.b + hk * a.v.h;
  const int c = threadIdx.x % PPR * EP;
  const int64_t live = pos < held ? pos : held;
  for (int64_t row = (int64_t)blockIdx.y * PER + threadIdx.x / PPR; row < live; row += (int64_t)gridDim.y * PER) {
    int64_t s = row;                                 // the token whose place this row is
    if (row >= a.sinks) {
      const int64_t r = row - a.sinks, ring = (int64_t)pos - a.sinks;
      s = a.sinks + ring - 1 - (ring - 1 - r) % a.window;   // (row < live: ring - 1 >= r or the ring is full)
    }
    const int64_t to = (bk * held + row) * D + c;
    *reinterpret_cast<u32x4*>(static_cast<E*>(a.kcache) + to) = *reinterpret_cast<const u32x4*>(k + s * a.k.t + c);
    *reinterpret_cast<u32x4*>(static_cast<E*>(a.vcache) + to) = *reinterpret_cast<const u32x4*>(v + s * a.v.t + c);
  }
  if (blockIdx.y == 0 && threadIdx.x == 0) a.pos[bk] = pos;
}

template <typename E, int D>
hipError_t launch_cache(const WindowCacheArgs& a, hipStream_t s) {
  constexpr int PER = 256 / (D * sizeof(E) / 16);
  int64_t held = (int64_t)a.sinks + a.window;
  if (held > a.L) held = a.L;
  int64_t y = (held + 4 * PER - 1) / (4 * PER);      // four rows a thread
  y = y < 1 ? 1 : y > 1024 ? 1024 : y;
  window_cache_kernel<E, D><<<dim3(a.B * a.Hkv, (unsigned)y), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// Workgroups per key/value head: two on every compute unit, as many as fit (a wave's trips to memory hide behind those of its
// neighbours; with one of four waves more, the join costs more than it brings: 96 -> 98 us at 256 heads of 4096 rows), as long
// as every wave has a tile.
int window_step_splits(int64_t heads, int64_t held, int rows) {
  const int64_t wgs = heads * ((rows + 31) / 32), tiles = (held + KT - 1) / KT + 1;
  int64_t n = (512 + wgs - 1) / wgs;
  if (n > (tiles + 3) / 4) n = (tiles + 3) / 4;
  return n < 1 ? 1 : n > 64 ? 64 : (int)n;
}

hipError_t launch_window_step(const WindowStepArgs& a, int d, bool bf16, hipStream_t s) {
  if (bf16) return d == 64 ? launch<MatBf16, 64>(a, s) : launch<MatBf16, 128>(a, s);
  return d == 64 ? launch<MatF32, 64>(a, s) : launch<MatF32, 128>(a, s);
}

hipError_t launch_window_cache(const WindowCacheArgs& a, int d, bool bf16, hipStream_t s) {
  if (bf16) return d == 64 ? launch_cache<uint16_t, 64>(a, s) : launch_cache<uint16_t, 128>(a, s);
  return d == 64 ? launch_cache<float, 64>(a, s) : launch_cache<float, 128>(a, s);
}

}  // namespace linattn
