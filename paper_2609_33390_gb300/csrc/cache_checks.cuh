// Checks of the context cache's calls that need no GPU, and pieces of their workspace's layout.
#pragma once

#include <math.h>

#include "cache.cuh"

namespace brisk {

constexpr size_t ALIGN = 256;
inline size_t up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
inline bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline size_t esize(int dt) { return dt == BRISK_DT_BF16 ? 2 : 4; }

inline bool dims_ok(const brisk_cache_dims* d) {
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
inline bool view_ok(const brisk_view* v, const brisk_cache_dims* d, long long seqs, long long toks, long long heads,
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

// Sizes of a call, before its work is divided.
inline AttendArgs undivided(const brisk_cache_dims* d) {
  AttendArgs a{};
  a.B = d->B; a.L = d->L; a.G = d->Hq / d->Hkv; a.Hkv = d->Hkv; a.D = d->D; a.P = d->P; a.S = d->S;
  a.dt = d->dtype;
  a.by_L.set(a.L);
  a.by_G.set(a.G);
  a.by_LG.set(a.L * a.G);
  return a;
}

struct CacheWs {
  size_t status, errs, cum, part_p, ml_p, part_o, ml_o, total;
};

// The workspace of an attention call whose work is divided.
inline CacheWs cache_ws(const AttendArgs& a) {
  CacheWs w{};
  const long long LG = a.L * a.G, R = a.B * LG;
  const long long tiles_p = a.P > 0 ? (R + a.sh.rt_p - 1) / a.sh.rt_p * a.Hkv : 0;
  const long long tiles_o = a.S > 0 ? (LG + a.sh.rt_o - 1) / a.sh.rt_o * a.Hkv * a.B : 0;
  const long long rows_p = (tiles_p + (a.sh.grid_p ? a.sh.grid_p : a.sh.grid_o)) * (R < a.sh.rt_p ? R : a.sh.rt_p);
  // (a unit may be of several key heads, each with slots of its own)
  const long long rows_o = (tiles_o + ((long long)a.sh.grid_o << a.sh.log_heads)) * (LG < a.sh.rt_o ? LG : a.sh.rt_o);
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t q = o; o = up(o + bytes); return q; };
  w.status = take(ALIGN);
  w.errs = take(sizeof(int32_t) * (a.sh.grid_p + a.sh.grid_o));
  w.cum = take(sizeof(int32_t) * (a.B + 1));
  w.ml_p = take(sizeof(float2) * rows_p);
  w.ml_o = take(sizeof(float2) * rows_o);
  w.part_p = take(sizeof(float) * rows_p * a.D);
  w.part_o = take(sizeof(float) * rows_o * a.D);
  w.total = o;
  return w;
}

// Whether attention's units of work, all caches full, are counted in 31 bits.
inline bool units_ok(const AttendArgs& a) {
  const long long LG = a.L * a.G, R = a.B * LG;
  const double pre = (double)a.Hkv * ((R + a.sh.rt_p - 1) / a.sh.rt_p) * a.sh.kP;
  const double own = (double)(a.Hkv >> a.sh.log_heads) * a.B * ((LG + a.sh.rt_o - 1) / a.sh.rt_o) * ((a.S + a.sh.kt - 1) / a.sh.kt);
  return pre + own < 2.0e9;
}

template <typename T>
inline T* at(void* base, size_t off) { return reinterpret_cast<T*>(static_cast<char*>(base) + off); }

inline void lay_out(AttendArgs* a, void* ws) {
  const CacheWs w = cache_ws(*a);
  a->part_p = at<float>(ws, w.part_p);
  a->part_o = at<float>(ws, w.part_o);
  a->ml_p = at<float2>(ws, w.ml_p);
  a->ml_o = at<float2>(ws, w.ml_o);
  a->cum = at<int32_t>(ws, w.cum);
  a->errs = at<int32_t>(ws, w.errs);
  a->status = at<int32_t>(ws, w.status);
}

// In the place of a scale of 0, which would make NaN of the masked scores' -inf: the smallest number above it (2^-149),
// with which every finite score is below 2^-21.
constexpr float SMALLEST_SCALE = 1.40129846e-45f;

// (kernels have scores in log2 units, in which the scale must be finite too: up to 2.35e38)
inline bool scale_ok(float s) { return s >= 0.f && isfinite(s * LOG2E); }

}  // namespace brisk
