// C ABI of attention over a shared prefix, the attention weights of own entries and the eviction by
// them: argument checks, workspace layout, launches.
#include <math.h>

#include "cache.cuh"

using namespace brisk;

namespace {

constexpr size_t ALIGN = 256;
inline size_t up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
inline bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline size_t esize(int dt) { return dt == BRISK_DT_BF16 ? 2 : 4; }

bool dims_ok(const brisk_cache_dims* d) {
  if (!d || d->B < 1 || d->B > CACHE_MAX_B || d->L < 1 || d->Hkv < 1 || d->Hq < d->Hkv || d->Hq % d->Hkv != 0)
    return false;
  if (d->D < 8 || d->D > CACHE_MAX_D || d->D % 8 != 0 || d->P < 0 || d->S < 0) return false;
  if (d->P > (1 << 30) || d->S > (1 << 30)) return false;
  if (d->dtype != BRISK_DT_F32 && d->dtype != BRISK_DT_BF16) return false;
  // query rows, and tiles of them over all keys, are counted in 32 and 62 bits
  return (long long)d->B * d->L <= (1 << 30) / d->Hq;
}

// Element strides of a tensor of the given extents: rows start on 16 bytes, no dimension runs
// backwards or stands still. An extent of one needs no stride (it is set to the row's).
bool view_ok(const brisk_view* v, const brisk_cache_dims* d, long long seqs, long long toks, long long heads,
             CacheView* out) {
  *out = CacheView{};
  if (seqs == 0 || toks == 0) return true;
  if (!v || !v->ptr || !aligned(v->ptr, 16)) return false;
  const long long ext[3] = {seqs, toks, heads}, in[3] = {v->seq, v->tok, v->head};
  long long s[3];
  const long long per16 = 16 / (long long)esize(d->dtype), most = (1LL << 39) / (long long)esize(d->dtype);
  for (int i = 0; i < 3; ++i) {
    s[i] = ext[i] > 1 ? in[i] : d->D;
    if (s[i] < d->D || s[i] % per16 != 0 || s[i] >= most) return false;
  }
  out->p = v->ptr;
  out->seq = s[0];
  out->tok = s[1];
  out->head = s[2];
  return true;
}

struct CacheWs {
  size_t status, errs, cum, part_p, ml_p, part_o, ml_o, total;
};

AttendArgs sizes_of(const brisk_cache_dims* d) {
  AttendArgs a{};
  a.B = d->B; a.L = d->L; a.G = d->Hq / d->Hkv; a.Hkv = d->Hkv; a.D = d->D; a.P = d->P; a.S = d->S;
  a.dt = d->dtype;
  a.by_L.set(a.L);
  a.by_G.set(a.G);
  a.by_LG.set(a.L * a.G);
  divide(&a);
  return a;
}

CacheWs cache_ws(const brisk_cache_dims* d) {
  CacheWs w{};
  const AttendArgs a = sizes_of(d);
  const long long LG = a.L * a.G, R = d->B * LG;
  const long long tiles_p = d->P > 0 ? (R + a.sh.rt_p - 1) / a.sh.rt_p * d->Hkv : 0;
  const long long tiles_o = d->S > 0 ? (LG + a.sh.rt_o - 1) / a.sh.rt_o * d->Hkv * d->B : 0;
  const long long rows_p = (tiles_p + (a.sh.grid_p ? a.sh.grid_p : a.sh.grid_o)) * (R < a.sh.rt_p ? R : a.sh.rt_p);
  const long long rows_o = (tiles_o + a.sh.grid_o) * (LG < a.sh.rt_o ? LG : a.sh.rt_o);
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t q = o; o = up(o + bytes); return q; };
  w.status = take(ALIGN);
  w.errs = take(sizeof(int32_t) * (a.sh.grid_p + a.sh.grid_o));
  w.cum = take(sizeof(int32_t) * (d->B + 1));
  w.ml_p = take(sizeof(float2) * rows_p);
  w.ml_o = take(sizeof(float2) * rows_o);
  w.part_p = take(sizeof(float) * rows_p * d->D);
  w.part_o = take(sizeof(float) * rows_o * d->D);
  w.total = o;
  return w;
}

// Whether attention's units of work, all caches full, are counted in 31 bits.
bool units_ok(const brisk_cache_dims* d) {
  const AttendArgs a = sizes_of(d);
  const long long LG = a.L * a.G, R = d->B * LG;
  const double pre = (double)d->Hkv * ((R + a.sh.rt_p - 1) / a.sh.rt_p) * ((d->P + a.sh.kt - 1) / a.sh.kt);
  const double own = (double)d->Hkv * d->B * ((LG + a.sh.rt_o - 1) / a.sh.rt_o) * ((d->S + a.sh.kt - 1) / a.sh.kt);
  return pre + own < 2.0e9;
}

// In the place of a scale of 0, which would make NaN of the masked scores' -inf: the smallest number above it (2^-149),
// with which every finite score is below 2^-21.
constexpr float SMALLEST = 1.40129846e-45f;

template <typename T>
inline T* at(void* base, size_t off) { return reinterpret_cast<T*>(static_cast<char*>(base) + off); }

// (kernels have scores in log2 units, in which the scale must be finite too: up to 2.35e38)
bool scale_ok(float s) { return s >= 0.f && isfinite(s * LOG2E); }

}  // namespace

extern "C" {

size_t brisk_cache_workspace_bytes(const brisk_cache_dims* dims) {
  return dims_ok(dims) ? cache_ws(dims).total : 0;
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
  if (!units_ok(d)) return BRISK_ERR_UNSUPPORTED;
  const CacheWs w = cache_ws(d);
  a.own_len = own_len;
  a.visible = visible;
  a.sl2 = scale * LOG2E;
  a.out = out;
  a.lse = lse;
  a.part_p = at<float>(ws, w.part_p);
  a.part_o = at<float>(ws, w.part_o);
  a.ml_p = at<float2>(ws, w.ml_p);
  a.ml_o = at<float2>(ws, w.ml_o);
  a.cum = at<int32_t>(ws, w.cum);
  a.errs = at<int32_t>(ws, w.errs);
  a.status = at<int32_t>(ws, w.status);
  a.wait_limit = wait_limit_cycles();
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a.sl2 == 0.f) a.sl2 = SMALLEST;
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
  if (!units_ok(d) || (long long)d->B * d->Hkv * ((d->S + 63) / 64) > 0x7fffffffLL) return BRISK_ERR_UNSUPPORTED;
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
  a.status = at<int32_t>(ws, cache_ws(d).status);
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
  a.status = at<int32_t>(ws, cache_ws(d).status);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return launch_evict(a, st) == cudaSuccess ? BRISK_OK : BRISK_ERR_CUDA;
}

}  // extern "C"
