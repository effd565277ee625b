// C ABI of attention over a shared prefix, the attention weights of own entries and the eviction by
// them: argument checks, workspace layout, launches.
#include "cache_checks.cuh"

using namespace brisk;

namespace {

AttendArgs sizes_of(const brisk_cache_dims* d) {
  AttendArgs a = undivided(d);
  divide(&a);
  return a;
}

}  // namespace

extern "C" {

size_t brisk_cache_workspace_bytes(const brisk_cache_dims* dims) {
  return dims_ok(dims) ? cache_ws(sizes_of(dims)).total : 0;
}

brisk_status brisk_prefix_attend(const brisk_cache_dims* d, const brisk_view* q, const brisk_view* k_prefix,
                                 const brisk_view* v_prefix, const brisk_view* k_own, const brisk_view* v_own,
                                 const int32_t* own_len, const int32_t* visible, float scale, void* out,
                                 float* lse, void* ws, void* stream) {
  if (!dims_ok(d) || !own_len || !out || !aligned(out, 16) || !ws || !aligned(ws, ALIGN) || !scale_ok(scale))
    return BRISK_ERR_INVALID_ARG;
  AttendArgs a = sizes_of(d);
  if (!view_ok(q, d, d->B, d->L, d->Hq, &a.q) || !view_ok(k_prefix, d, 1, d->P, d->Hkv, &a.kp) ||
      !view_ok(v_prefix, d, 1, d->P, d->Hkv, &a.vp) || !view_ok(k_own, d, d->B, d->S, d->Hkv, &a.ko) ||
      !view_ok(v_own, d, d->B, d->S, d->Hkv, &a.vo))
    return BRISK_ERR_INVALID_ARG;
  if (!units_ok(a)) return BRISK_ERR_UNSUPPORTED;
  a.own_len = own_len;
  a.visible = visible;
  a.sl2 = scale * LOG2E;
  a.out = out;
  a.lse = lse;
  lay_out(&a, ws);
  a.wait_limit = wait_limit_cycles();
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a.sl2 == 0.f) a.sl2 = SMALLEST_SCALE;
  if ((d->dtype == BRISK_DT_BF16 ? launch_attend_tc(a, st) : launch_attend_f32(a, st)) != cudaSuccess)
    return BRISK_ERR_CUDA;
  if (launch_merge(a, st) != cudaSuccess) return BRISK_ERR_CUDA;
  return BRISK_OK;
}

brisk_status brisk_cache_weights(const brisk_cache_dims* d, const brisk_view* q, const float* lse,
                                 const brisk_view* k_own, const int32_t* own_len, const int32_t* visible,
                                 float scale, float decay, const float* acc_in, float* acc_out, void* ws,
                                 void* stream) {
  if (!dims_ok(d) || !lse || !own_len || (d->S > 0 && !acc_out) || !ws || !aligned(ws, ALIGN) ||
      !scale_ok(scale) || !isfinite(decay))
    return BRISK_ERR_INVALID_ARG;
  WeightArgs a{};
  if (!view_ok(q, d, d->B, d->L, d->Hq, &a.q) || !view_ok(k_own, d, d->B, d->S, d->Hkv, &a.ko))
    return BRISK_ERR_INVALID_ARG;
  // one CTA a key tile: their number is a grid's first dimension
  if (!units_ok(sizes_of(d)) || (long long)d->B * d->Hkv * ((d->S + 63) / 64) > 0x7fffffffLL) return BRISK_ERR_UNSUPPORTED;
  a.B = d->B; a.L = d->L; a.G = d->Hq / d->Hkv; a.Hkv = d->Hkv; a.D = d->D; a.S = d->S; a.dt = d->dtype;
  a.by_G.set(a.G);
  a.own_len = own_len;
  a.visible = visible;
  a.lse = lse;
  a.scale = scale;
  a.sl2 = scale * LOG2E;
  a.decay = decay;
  a.acc_in = acc_in;
  a.acc_out = acc_out;
  a.status = at<int32_t>(ws, cache_ws(sizes_of(d)).status);
  a.wait_limit = wait_limit_cycles();
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (d->S == 0 || d->dtype == BRISK_DT_BF16)   // (the fp32 kernel writes the word itself)
    if (cudaMemsetAsync(a.status, 0, sizeof(int32_t), st) != cudaSuccess) return BRISK_ERR_CUDA;
  if (d->S == 0) return BRISK_OK;
  divide(&a);
  return (d->dtype == BRISK_DT_BF16 ? launch_weights_tc(a, st) : launch_weights_f32(a, st)) == cudaSuccess
             ? BRISK_OK : BRISK_ERR_CUDA;
}

brisk_status brisk_cache_evict(const brisk_cache_dims* d, const brisk_view* k, const brisk_view* v,
                               const float* acc, const int32_t* own_len, int32_t keep, int32_t recent,
                               const brisk_view* k_to, const brisk_view* v_to, float* acc_to,
                               int32_t* len_to, int32_t* kept, void* ws, void* stream) {
  if (!dims_ok(d) || keep < 1 || keep > (1 << 30) || recent < 0 || recent > keep || (d->S > 0 && !acc) ||
      !own_len || !acc_to || !len_to || !kept || !ws || !aligned(ws, ALIGN))
    return BRISK_ERR_INVALID_ARG;
  EvictArgs a{};
  if (!view_ok(k, d, d->B, d->S, d->Hkv, &a.k) || !view_ok(v, d, d->B, d->S, d->Hkv, &a.v) ||
      !view_ok(k_to, d, d->B, keep, d->Hkv, &a.k_to) || !view_ok(v_to, d, d->B, keep, d->Hkv, &a.v_to))
    return BRISK_ERR_INVALID_ARG;
  // entries move between buffers: a place may be written before it is read
  const void *from[2] = {a.k.p, a.v.p}, *to[2] = {a.k_to.p, a.v_to.p};
  for (const void* f : from)
    for (const void* t : to)
      if (f == t) return BRISK_ERR_INVALID_ARG;
  if (acc == acc_to || own_len == len_to || a.k_to.p == a.v_to.p) return BRISK_ERR_INVALID_ARG;
  // a sequence's 16-byte pieces, and the kernel that moves them one beyond its last CTA, in 31 bits
  const double vecs = (double)keep * d->Hkv * (d->D * (double)esize(d->dtype) / 16);
  if (vecs >= 2.0e9) return BRISK_ERR_UNSUPPORTED;
  a.B = d->B; a.Hkv = d->Hkv; a.D = d->D; a.S = d->S; a.dt = d->dtype; a.keep = keep; a.recent = recent;
  a.acc = acc;
  a.own_len = own_len;
  a.acc_to = acc_to;
  a.len_to = len_to;
  a.kept = kept;
  a.status = at<int32_t>(ws, cache_ws(sizes_of(d)).status);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return launch_evict(a, st) == cudaSuccess ? BRISK_OK : BRISK_ERR_CUDA;
}

}  // extern "C"
