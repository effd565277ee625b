// C ABI of the context cache in 4 bits: argument checks, launches.
#include "cache_checks.cuh"
#include "packed.cuh"

using namespace brisk;

namespace {

bool packed_dims_ok(const brisk_cache_dims* d) { return dims_ok(d) && d->D % GROUP == 0; }

AttendArgs sizes_of(const brisk_cache_dims* d) {
  AttendArgs a = undivided(d);
  divide_packed(&a);
  return a;
}

// Byte strides of codes or scales of the given extents: rows of `row` bytes that start on `step` bytes.
bool strides_ok(const void* ptr, const int64_t (&in)[3], const long long (&ext)[3], int row, int step, long long (&out)[3]) {
  if (!ptr || !aligned(ptr, step)) return false;
  for (int i = 0; i < 3; ++i) {
    out[i] = ext[i] > 1 ? in[i] : row;
    if (out[i] < row || out[i] % step != 0 || out[i] >= (1LL << (i == 1 ? 32 : 39))) return false;
  }
  return true;
}
bool packed_ok(const brisk_packed* v, const brisk_cache_dims* d, PackedView* out) {
  *out = PackedView{};
  if (d->S == 0) return true;
  if (!v) return false;
  const long long ext[3] = {d->B, d->S, d->Hkv};
  const int64_t codes[3] = {v->seq, v->tok, v->head}, scales[3] = {v->scale_seq, v->scale_tok, v->scale_head};
  long long c[3], s[3];
  if (!strides_ok(v->codes, codes, ext, d->D / 2, d->D % 32 == 0 ? 16 : 8, c) ||
      !strides_ok(v->scales, scales, ext, scale_row(d->D), scale_row(d->D), s))
    return false;
  *out = PackedView{static_cast<uint8_t*>(v->codes), static_cast<uint8_t*>(v->scales), c[0], c[2], s[0], s[2], (uint32_t)c[1], (uint32_t)s[1]};
  return true;
}

brisk_status move_args(const brisk_cache_dims* d, int32_t T, const brisk_view* k, const brisk_view* v, const int32_t* start,
                       const int32_t* count, const brisk_packed* kp, const brisk_packed* vp, void* ws, PackedMoveArgs* a) {
  if (!packed_dims_ok(d) || T < 1 || T > (1 << 30) || !start || !ws || !aligned(ws, ALIGN)) return BRISK_ERR_INVALID_ARG;
  CacheView ck, cv;
  if (!view_ok(k, d, d->B, T, d->Hkv, &ck) || !view_ok(v, d, d->B, T, d->Hkv, &cv) || !packed_ok(kp, d, &a->kp) ||
      !packed_ok(vp, d, &a->vp))
    return BRISK_ERR_INVALID_ARG;
  const int pieces = d->D * (int)esize(d->dtype) / 16;
  // tokens that a grid's dimensions do not take
  if ((double)d->Hkv * pieces > 65535.0 * 256) return BRISK_ERR_UNSUPPORTED;
  a->B = d->B; a->T = T; a->Hkv = d->Hkv; a->D = d->D; a->S = d->S; a->dt = d->dtype;
  a->by_row.set(pieces);
  a->by_token.set(d->Hkv * pieces);
  a->step = d->Hkv * pieces < 256 ? 256 / (d->Hkv * pieces) : 1;
  a->k = ck;
  a->v = cv;
  a->start = start;
  a->count = count;
  a->status = static_cast<int32_t*>(ws);           // (the workspace's first word, as of every call)
  return BRISK_OK;
}

}  // namespace

extern "C" {

size_t brisk_packed_workspace_bytes(const brisk_cache_dims* dims) {
  return packed_dims_ok(dims) ? cache_ws(sizes_of(dims)).total : 0;
}

brisk_status brisk_packed_store(const brisk_cache_dims* d, int32_t T, const brisk_view* k, const brisk_view* v,
                                const int32_t* start, const int32_t* count, const brisk_packed* k_to,
                                const brisk_packed* v_to, void* ws, void* stream) {
  PackedMoveArgs a{};
  const brisk_status s = move_args(d, T, k, v, start, count, k_to, v_to, ws, &a);
  if (s != BRISK_OK) return s;
  if (d->S > 0 && (a.kp.codes == a.vp.codes || a.kp.scales == a.vp.scales)) return BRISK_ERR_INVALID_ARG;
  return launch_packed_store(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? BRISK_OK : BRISK_ERR_CUDA;
}

brisk_status brisk_packed_load(const brisk_cache_dims* d, int32_t T, const brisk_packed* k, const brisk_packed* v,
                               const int32_t* start, const int32_t* count, const brisk_view* k_to, const brisk_view* v_to,
                               void* ws, void* stream) {
  PackedMoveArgs a{};
  const brisk_status s = move_args(d, T, k_to, v_to, start, count, k, v, ws, &a);
  if (s != BRISK_OK) return s;
  if (a.k.p == a.v.p) return BRISK_ERR_INVALID_ARG;
  return launch_packed_load(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? BRISK_OK : BRISK_ERR_CUDA;
}

brisk_status brisk_packed_attend(const brisk_cache_dims* d, const brisk_view* q, const brisk_view* k_prefix,
                                 const brisk_view* v_prefix, const brisk_packed* k_own, const brisk_packed* v_own,
                                 const int32_t* own_len, const int32_t* visible, float scale, void* out, float* lse,
                                 void* ws, void* stream) {
  if (!packed_dims_ok(d) || !own_len || !out || !aligned(out, 16) || !ws || !aligned(ws, ALIGN) || !scale_ok(scale))
    return BRISK_ERR_INVALID_ARG;
  PackedArgs p{};
  p.a = sizes_of(d);
  AttendArgs& a = p.a;
  if (!view_ok(q, d, d->B, d->L, d->Hq, &a.q) || !view_ok(k_prefix, d, 1, d->P, d->Hkv, &a.kp) ||
      !view_ok(v_prefix, d, 1, d->P, d->Hkv, &a.vp) || !packed_ok(k_own, d, &p.k) || !packed_ok(v_own, d, &p.v))
    return BRISK_ERR_INVALID_ARG;
  if (!units_ok(a)) return BRISK_ERR_UNSUPPORTED;
  a.own_len = own_len;
  a.visible = visible;
  a.sl2 = scale * LOG2E;
  if (a.sl2 == 0.f) a.sl2 = SMALLEST_SCALE;
  a.out = out;
  a.lse = lse;
  lay_out(&a, ws);
  a.wait_limit = wait_limit_cycles();
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = a.sh.rt_o == SLOT_ROWS ? launch_packed_tc(p, st) : launch_packed_few(p, st);
  if (e == cudaSuccess && d->P > 0) e = d->dtype == BRISK_DT_BF16 ? launch_prefix_tc(a, st) : launch_prefix_f32(a, st);
  if (e == cudaSuccess) e = launch_merge(a, st);
  return e == cudaSuccess ? BRISK_OK : BRISK_ERR_CUDA;
}

}  // extern "C"
