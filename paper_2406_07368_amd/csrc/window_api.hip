// C ABI of softmax attention over a sliding window with sinks (include/linattn.h): argument validation, launch planning.
#include "../../include/linattn.h"

#include <hip/hip_runtime.h>

#include "common.h"
#include "rows.h"
#include "window.h"

using namespace linattn;

namespace {

linattn_status check(const linattn_window_desc* d, int32_t L) {
  if (!d) return LINATTN_ERR_NULL;
  if (d->io_dtype != LINATTN_F32 && d->io_dtype != LINATTN_BF16) return LINATTN_ERR_DTYPE;
  if (d->B < 1 || d->H < 1 || d->H_kv < 1 || d->H % d->H_kv || (int64_t)d->B * d->H > (int64_t)1 << 20) return LINATTN_ERR_SHAPE;
  if (d->d != 64 && d->d != 128) return LINATTN_ERR_SHAPE;
  if (d->window < 1 || d->sinks < 0 || d->sinks > LINATTN_MAX_SINKS) return LINATTN_ERR_SHAPE;
  if (!finite(d->scale) || d->scale < 0.f) return LINATTN_ERR_SHAPE;
  if (L < 0 || L > kMaxTokens || (int64_t)d->B * d->H * ((L + 127) / 128) > (int64_t)1 << 23) return LINATTN_ERR_SHAPE;   // (a grid's limit)
  return LINATTN_OK;
}
linattn_status check_rows(const linattn_window_desc* d, int32_t L, bool gradient) {
  bool ok = good_input(d->q, d->B, d->H, L) && good_input(d->k, d->B, d->H_kv, L) && good_input(d->v, d->B, d->H_kv, L);
  if (gradient)
    ok = ok && good_input(d->out, d->B, d->H, L) && good_input(d->dout, d->B, d->H, L) && good_output(d->dq, d->B, d->H, L, d->d) &&
         good_output(d->dk, d->B, d->H_kv, L, d->d) && good_output(d->dv, d->B, d->H_kv, L, d->d);
  else
    ok = ok && good_output(d->out, d->B, d->H, L, d->d);
  return ok ? LINATTN_OK : LINATTN_ERR_SHAPE;
}

linattn_status check_step(const linattn_window_desc* d, int32_t kk) {
  const linattn_status st = check(d, 0);
  if (st != LINATTN_OK) return st;
  if (kk < 1 || kk > LINATTN_MAX_DRAFT || (int64_t)(d->H / d->H_kv) * kk > (int64_t)1 << 20) return LINATTN_ERR_SHAPE;   // (a grid's limit)
  return LINATTN_OK;
}

WindowArgs args(const linattn_window_desc* d, int32_t L, const void* q, const void* k, const void* v, const int32_t* lens) {
  WindowArgs a{};
  a.q = rows(q, d->q); a.k = rows(k, d->k); a.v = rows(v, d->v);
  a.lens = lens; a.B = d->B; a.H = d->H; a.Hkv = d->H_kv; a.L = L;
  a.window = d->window; a.sinks = d->sinks; a.scale = d->scale;
  return a;
}

struct GradientPlan {
  int far, parts;                                 // see WindowArgs
  size_t off_sinks, off_part, bytes;
};
size_t round256(size_t x) { return (x + 255) / 256 * 256; }
GradientPlan plan_gradient(const linattn_window_desc* d, int32_t L) {
  GradientPlan p{};
  const int64_t heads = (int64_t)d->B * d->H_kv, group = d->H / d->H_kv;
  const int tiles = (L + kWindowQ - 1) / kWindowQ, near = window_far_tile(d->window) < tiles ? window_far_tile(d->window) : tiles;
  // few key tiles: as many workgroups for each as the chip has room for, with four query tiles each or more
  const int64_t wgs = heads * ((L + kWindowKeys - 1) / kWindowKeys);
  int64_t parts = 256 / wgs < near * group / 4 ? 256 / wgs : near * group / 4;
  p.parts = parts < 1 ? 1 : (int)parts;
  if (d->sinks > 0 && tiles > near) {
    const int64_t items = (int64_t)(tiles - near) * group;
    int64_t n = (512 + heads - 1) / heads;
    if (n > (items + 3) / 4) n = (items + 3) / 4;
    p.far = (int)n;
  }
  p.off_sinks = round256(2 * (size_t)d->B * d->H * L * sizeof(float));
  p.off_part = p.off_sinks + round256(p.far ? (size_t)heads * (p.parts + 2 * p.far) * 2 * d->sinks * d->d * sizeof(float) : 0);
  p.bytes = p.off_part + (p.parts > 1 ? (size_t)heads * p.parts * 2 * L * d->d * sizeof(float) : 0);
  return p;
}

}  // namespace

extern "C" {

linattn_status linattn_window_prefill(const linattn_window_desc* desc, int32_t L, const void* q, const void* k, const void* v,
                                      const int32_t* lens, void* out, float* lse, void* kcache, void* vcache, int32_t* pos,
                                      void* hip_stream) {
  linattn_status st = check(desc, L);
  if (st == LINATTN_OK) st = check_rows(desc, L, false);
  if (st != LINATTN_OK) return st;
  if (L > 0 && (!q || !k || !v || !out)) return LINATTN_ERR_NULL;
  const int cache = (kcache != nullptr) + (vcache != nullptr) + (pos != nullptr);
  if (cache != 0 && cache != 3) return LINATTN_ERR_NULL;
  if (!aligned16_all({q, k, v, lens, out, lse, kcache, vcache, pos})) return LINATTN_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool bf16 = desc->io_dtype == LINATTN_BF16;
  hipError_t e = hipSuccess;
  if (L > 0) {
    WindowArgs a = args(desc, L, q, k, v, lens);
    a.out = rows(out, desc->out); a.lse = lse;
    e = bf16 ? launch_window_prefill_bf16(a, desc->d, s) : launch_window_prefill_f32(a, desc->d, s);
  }
  if (e == hipSuccess && cache) {
    WindowCacheArgs c{rows(k, desc->k), rows(v, desc->v), lens, kcache, vcache, pos, desc->B, desc->H_kv, L, desc->window, desc->sinks};
    e = launch_window_cache(c, desc->d, bf16, s);
  }
  return e == hipSuccess ? LINATTN_OK : LINATTN_ERR_HIP;
}

size_t linattn_window_backward_workspace_bytes(const linattn_window_desc* desc, int32_t L) {
  return check(desc, L) == LINATTN_OK && desc->io_dtype == LINATTN_BF16 && L > 0 ? plan_gradient(desc, L).bytes : 0;
}

linattn_status linattn_window_backward(const linattn_window_desc* desc, int32_t L, const void* q, const void* k, const void* v,
                                       const int32_t* lens, const void* out, const float* lse, const void* dout, void* dq, void* dk,
                                       void* dv, void* workspace, size_t workspace_bytes, void* hip_stream) {
  linattn_status st = check(desc, L);
  if (st == LINATTN_OK) st = check_rows(desc, L, true);
  if (st != LINATTN_OK) return st;
  if (desc->io_dtype != LINATTN_BF16) return LINATTN_ERR_UNSUPPORTED;
  if (L > 0 && (!q || !k || !v || !out || !lse || !dout || !dq || !dk || !dv)) return LINATTN_ERR_NULL;
  if (!aligned16_all({q, k, v, lens, out, lse, dout, dq, dk, dv, workspace})) return LINATTN_ERR_ALIGN;
  if (L == 0) return LINATTN_OK;
  const GradientPlan p = plan_gradient(desc, L);
  if (!workspace || workspace_bytes < p.bytes) return LINATTN_ERR_WORKSPACE;
  WindowArgs a = args(desc, L, q, k, v, lens);
  a.out = rows(out, desc->out); a.dout = rows(dout, desc->dout);
  a.dq = rows(dq, desc->dq); a.dk = rows(dk, desc->dk); a.dv = rows(dv, desc->dv);
  a.lse = const_cast<float*>(lse);
  a.stats = static_cast<float*>(workspace);
  a.sink_part = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + p.off_sinks);
  a.part = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + p.off_part);
  a.far = p.far; a.parts = p.parts;
  a.dk_scale = L == 1 || (desc->window == 1 && desc->sinks == 0) ? 0.f : desc->scale;
  return launch_window_backward(a, desc->d, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? LINATTN_OK : LINATTN_ERR_HIP;
}

size_t linattn_window_step_workspace_bytes(const linattn_window_desc* desc, int32_t kk) {
  if (check_step(desc, kk) != LINATTN_OK) return 0;
  const int64_t heads = (int64_t)desc->B * desc->H_kv, R = (int64_t)(desc->H / desc->H_kv) * kk;
  const int n = window_step_splits(heads, (int64_t)desc->sinks + desc->window, (int)R);
  return n > 1 ? (size_t)heads * n * R * (desc->d + 2) * sizeof(float) : 0;
}

linattn_status linattn_window_step(const linattn_window_desc* desc, int32_t kk, const void* q, const void* k, const void* v,
                                   void* kcache, void* vcache, int32_t* pos, const int32_t* n_commit, void* out, void* workspace,
                                   size_t workspace_bytes, void* hip_stream) {
  const linattn_status st = check_step(desc, kk);
  if (st != LINATTN_OK) return st;
  if (!q || !k || !v || !kcache || !vcache || !pos || !out) return LINATTN_ERR_NULL;
  if (!aligned16_all({q, k, v, kcache, vcache, pos, n_commit, out, workspace})) return LINATTN_ERR_ALIGN;
  const size_t need = linattn_window_step_workspace_bytes(desc, kk);
  if (need && (!workspace || workspace_bytes < need)) return LINATTN_ERR_WORKSPACE;
  WindowStepArgs a{};
  a.q = q; a.k = k; a.v = v; a.kcache = kcache; a.vcache = vcache; a.pos = pos; a.n_commit = n_commit; a.out = out;
  a.ws = static_cast<float*>(workspace);
  a.B = desc->B; a.H = desc->H; a.Hkv = desc->H_kv; a.kk = kk; a.window = desc->window; a.sinks = desc->sinks; a.scale = desc->scale;
  a.nsplit = window_step_splits((int64_t)a.B * a.Hkv, (int64_t)a.sinks + a.window, a.H / a.Hkv * kk);
  return launch_window_step(a, desc->d, desc->io_dtype == LINATTN_BF16, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? LINATTN_OK : LINATTN_ERR_HIP;
}

}  // extern "C"
