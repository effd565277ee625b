// Entries written into a cache in 4 bits, and read back.
//
// A thread has 16 bytes of an unquantised row (8 channels of bf16, 4 of fp32), so that every access of a warp, on
// either side, is a run of whole rows; the lanes of a group of 16 channels find its largest magnitude together. Both
// kernels are bound by the rows' bytes.
#include "packed.cuh"

namespace brisk {
namespace {

constexpr int MOVE_THREADS = 256, EACH = 4;        // pieces of a thread, whose loads are on their way together

__device__ __forceinline__ int rows_of(const PackedMoveArgs& a, int b, int* start, bool* bad) {
  const int first = a.start[b], n = a.count ? a.count[b] : a.T;
  *start = first;
  *bad = n < 0 || n > a.T || (n > 0 && (first < 0 || (long long)first + n > a.S));
  return min(max(n, 0), a.T);
}

template <typename T> constexpr int channels() { return 16 / (int)sizeof(T); }

template <typename T>
__global__ void __launch_bounds__(MOVE_THREADS) store_kernel(const __grid_constant__ PackedMoveArgs a) {
  constexpr int C = channels<T>(), LANES = GROUP / C;      // channels of a thread, threads of a group
  const int b = blockIdx.y;
  int start;
  bool bad;
  const int n = rows_of(a, b, &start, &bad);
  int code = bad ? BRISK_ERR_INVALID_ARG : BRISK_OK;
  const int e0 = (int)blockIdx.x * MOVE_THREADS * EACH + threadIdx.x;
  uint4 x[EACH];
  int t[EACH], h[EACH], c[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    // (the keys' pieces, then the values')
    int e = e0 + j * MOVE_THREADS;
    const bool value = e >= a.all;
    if (value) e -= a.all;
    const int row = a.by_piece.of(e);
    t[j] = a.by_heads.of(row);
    h[j] = row - t[j] * a.Hkv;
    c[j] = (e - row * a.by_piece.d) * C;
    const bool there = e < a.all && t[j] < n;
    const CacheView& from = value ? a.v : a.k;
    x[j] = make_uint4(0, 0, 0, 0);
    if (there) x[j] = ld_stream_v4(static_cast<const T*>(from.p) + b * from.seq + t[j] * from.tok + h[j] * from.head + c[j]);
    if (!there || start + (long long)t[j] < 0 || start + (long long)t[j] >= a.S) t[j] = -1;
    if (value) c[j] = ~c[j];
  }
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    float f[C];
    unpack(x[j], f, T());
    uint32_t top = 0;                              // magnitudes compare as their bits do, infinities and NaN on top
#pragma unroll
    for (int i = 0; i < C; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
    const bool odd = top >= 0x7f800000u;           // an infinity or NaN
    if (odd) {
      top = 0;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        f[i] = f[i] != f[i] ? 0.f : fminf(fmaxf(f[i], -3.4e38f), 3.4e38f);
        top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
      }
      if (t[j] >= 0) code = max(code, (int)BRISK_ERR_NUMERIC);
    }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = max(top, __shfl_xor_sync(FULL_MASK, top, o));
    const uint32_t byte = scale_byte(__uint_as_float(top));
    const float s = scale_value(byte), r = 1.f / s;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < C; i += 2) codes |= to_codes(quotient(f[i], s, r), quotient(f[i + 1], s, r)) << (4 * i);
    if (t[j] < 0) continue;
    const bool value = c[j] < 0;
    const int ch = value ? ~c[j] : c[j];
    const PackedView& to = value ? a.vp : a.kp;
    const long long at = start + (long long)t[j];
    uint8_t* row = to.codes + b * to.seq + at * to.tok + h[j] * to.head + ch / 2;
    if constexpr (C == 8) *reinterpret_cast<uint32_t*>(row) = codes;
    else *reinterpret_cast<uint16_t*>(row) = (uint16_t)codes;
    if (ch % GROUP == 0) to.scales[b * to.sseq + at * to.stok + h[j] * to.shead + ch / GROUP] = (uint8_t)byte;
  }
  if (a.alone) {
    code = __syncthreads_or(code == BRISK_ERR_NUMERIC) ? BRISK_ERR_NUMERIC : (bad ? BRISK_ERR_INVALID_ARG : BRISK_OK);
    if (threadIdx.x == 0) *a.status = code;
  } else if (code != BRISK_OK) {
    atomicMax(a.status, code);                     // (cleared before; the largest, whatever the order)
  }
}

template <typename T>
__global__ void __launch_bounds__(MOVE_THREADS) load_kernel(const __grid_constant__ PackedMoveArgs a) {
  constexpr int C = channels<T>();
  const int b = blockIdx.y;
  int start;
  bool bad;
  const int n = rows_of(a, b, &start, &bad);
  if (blockIdx.x == 0 && b == 0) {                 // the call's status: rows asked for that no cache has
    bool any = false;
    for (int i = threadIdx.x; i < a.B; i += MOVE_THREADS) {
      int s;
      bool x;
      rows_of(a, i, &s, &x);
      any |= x;
    }
    any = __syncthreads_or(any);
    if (threadIdx.x == 0) *a.status = any ? BRISK_ERR_INVALID_ARG : BRISK_OK;
  }
  const int e0 = (int)blockIdx.x * MOVE_THREADS * EACH + threadIdx.x;
  uint32_t codes[EACH], byte[EACH];
  T* to[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    int e = e0 + j * MOVE_THREADS;
    const bool value = e >= a.all;
    if (value) e -= a.all;
    const int row = a.by_piece.of(e), t = a.by_heads.of(row), h = row - t * a.Hkv, c = (e - row * a.by_piece.d) * C;
    const CacheView& out = value ? a.v : a.k;
    const PackedView& from = value ? a.vp : a.kp;
    const long long at = start + (long long)t;
    to[j] = nullptr;
    codes[j] = byte[j] = 0;
    if (e >= a.all) continue;
    to[j] = static_cast<T*>(const_cast<void*>(out.p)) + b * out.seq + t * out.tok + h * out.head + c;
    if (t >= n || at < 0 || at >= a.S) continue;
    const uint8_t* p = from.codes + b * from.seq + at * from.tok + h * from.head + c / 2;
    if constexpr (C == 8) codes[j] = __ldg(reinterpret_cast<const uint32_t*>(p));
    else codes[j] = __ldg(reinterpret_cast<const uint16_t*>(p));
    byte[j] = __ldg(from.scales + b * from.sseq + at * from.stok + h * from.shead + c / GROUP);
  }
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    if (!to[j]) continue;
    uint32_t x[4];
    from_codes(codes[j], x);
    const uint32_t s = scale_f16(byte[j]);
    float f[C];
#pragma unroll
    for (int i = 0; i < C / 2; ++i) {              // (the products are exact, in fp16 and in T)
      const uint32_t y = mul_f16(x[i], s);
      const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&y));
      f[2 * i] = z.x;
      f[2 * i + 1] = z.y;
    }
#pragma unroll
    for (int i = 0; i < C; i += 4) {
      if constexpr (C == 4) {
        __stcs(reinterpret_cast<float4*>(to[j]), make_float4(f[0], f[1], f[2], f[3]));
      } else if (i == 0) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const __nv_bfloat162 y = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
          w[k] = *reinterpret_cast<const uint32_t*>(&y);
        }
        __stcs(reinterpret_cast<uint4*>(to[j]), make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
  }
}

dim3 grid_of(const PackedMoveArgs& a) {
  const long long each = MOVE_THREADS * EACH;
  return dim3((unsigned)((2LL * a.all + each - 1) / each), a.B);
}

}  // namespace

cudaError_t launch_packed_store(const PackedMoveArgs& args, cudaStream_t stream) {
  PackedMoveArgs a = args;
  const dim3 grid = grid_of(a);
  a.alone = grid.x == 1 && grid.y == 1;
  cudaError_t e = a.alone ? cudaSuccess : cudaMemsetAsync(a.status, 0, sizeof(int32_t), stream);
  if (e != cudaSuccess) return e;
  if (a.dt == BRISK_DT_BF16) store_kernel<__nv_bfloat16><<<grid, MOVE_THREADS, 0, stream>>>(a);
  else store_kernel<float><<<grid, MOVE_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_packed_load(const PackedMoveArgs& a, cudaStream_t stream) {
  const dim3 grid = grid_of(a);
  if (a.dt == BRISK_DT_BF16) load_kernel<__nv_bfloat16><<<grid, MOVE_THREADS, 0, stream>>>(a);
  else load_kernel<float><<<grid, MOVE_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace brisk
