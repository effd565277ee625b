// Entries written into a cache in 4 bits, and read back.
//
// A thread has 16 bytes of an unquantised row (8 channels of bf16, 4 of fp32) at one place of a token, of EACH tokens'
// keys and values in turn (see tokens_each), so that every access of a warp, on either side, is a run of whole rows, and
// places are worked out once a thread. The lanes of a group of 16 channels find its largest magnitude together.
// Both are bound by the rows' bytes as soon as these are many: 16 times 4096 rows of 8 heads of 128, 336 MB, are written
// in 60 us (5.6 TB/s; the instructions, some 90 a piece, fill two thirds of the slots) and read back in 56 (6.0 TB/s).
// Few rows are bound by latency: lengths, rows, the scale's chain, 4 us.
#include <climits>

#include "packed.cuh"

namespace brisk {
namespace {

constexpr int MOVE_THREADS = 256;

__device__ __forceinline__ int rows_of(const PackedMoveArgs& a, int b, int* start, bool* bad) {
  const int first = a.start[b], n = a.count ? a.count[b] : a.T;
  *start = first;
  *bad = n < 0 || n > a.T || (n > 0 && (first < 0 || (long long)first + n > a.S));
  return min(max(n, 0), a.T);
}

template <typename T> constexpr int channels() { return 16 / (int)sizeof(T); }

// A thread's place: its first token and key head, its channel; `there`: it has one.
template <typename T, int EACH>
struct Place {
  int t, h, c;
  bool there;
  __device__ __forceinline__ Place(const PackedMoveArgs& a) {
    const int q = (int)blockIdx.z * MOVE_THREADS + threadIdx.x, r = a.by_token.of(q), e = q - r * a.by_token.d;
    h = a.by_row.of(e);
    c = (e - h * a.by_row.d) * channels<T>();
    // (tokens that need several CTAs: blockIdx.z counts these)
    there = a.by_token.d > MOVE_THREADS ? r == 0 : r < a.step;
    t = (int)blockIdx.x * EACH * a.step + (a.by_token.d > MOVE_THREADS ? 0 : r);
  }
};
// Which rows of a thread, counted from its first token's, are there and have a place in the cache.
struct Inside {
  int from;
  uint32_t n;
  __device__ __forceinline__ Inside(const PackedMoveArgs& a, int start, int rows, bool there, int t) {
    const int low = start < 0 ? (start == INT_MIN ? INT_MAX : -start) : 0;
    const int high = (int)min((long long)rows, (long long)a.S - start);
    from = t - low;
    n = there && high > low ? (uint32_t)(high - low) : 0;
  }
  __device__ __forceinline__ bool operator()(int on) const { return (uint32_t)(from + on) < n; }
};
// A thread's address in a tensor, `t` tokens on.
__device__ __forceinline__ const char* row_at(const CacheView& v, int es, int b, int h, int c, int t) {
  return static_cast<const char*>(v.p) + (b * v.seq + h * v.head + c + t * v.tok) * es;
}

// (Four tokens a thread: with 64 registers there are four CTAs an SM, not three: 16 prompts 51.7 -> 43.7 us.)
template <typename T, int EACH>
__global__ void __launch_bounds__(MOVE_THREADS, EACH == 4 ? 4 : 1) store_kernel(const __grid_constant__ PackedMoveArgs a) {
  constexpr int C = channels<T>(), LANES = GROUP / C;      // channels of a thread, threads of a group
  const int b = blockIdx.y;
  int start;
  bool bad;
  const int n = rows_of(a, b, &start, &bad);
  // rows of a padded batch that are not there (16 prompts of 1500 to 4096: written and read back in 119 us with what they took, 107 without)
  if ((int)blockIdx.x * EACH * a.step >= n && !bad && !a.alone) return;
  const Place<T, EACH> at(a);
  const Inside in(a, start, n, at.there, at.t);
  uint4 x[2][EACH];
  {
    const char *k = row_at(a.k, sizeof(T), b, at.h, at.c, at.t), *v = row_at(a.v, sizeof(T), b, at.h, at.c, at.t);
    const long long ks = a.step * a.k.tok * (long long)sizeof(T), vs = a.step * a.v.tok * (long long)sizeof(T);
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      x[0][j] = x[1][j] = make_uint4(0, 0, 0, 0);
      if (in(j * a.step)) {
        x[0][j] = ld_stream_v4(k + j * ks);
        x[1][j] = ld_stream_v4(v + j * vs);
      }
    }
  }
  const long long first = start + (long long)at.t;
  int code = bad ? BRISK_ERR_INVALID_ARG : BRISK_OK;
#pragma unroll
  for (int value = 0; value < 2; ++value) {
    const PackedView& to = value ? a.vp : a.kp;
    uint8_t* codes = to.codes + b * to.seq + at.h * to.head + at.c / 2 + first * to.tok;
    uint8_t* scales = to.scales + b * to.sseq + at.h * to.shead + at.c / GROUP + first * to.stok;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const uint4 y = x[value][j];
      const uint32_t w[4] = {y.x, y.y, y.z, y.w};
      float f[C];
      unpack(y, f, T());
      uint32_t top = 0;                            // magnitudes compare as their bits do, infinities and NaN on top
      if constexpr (C == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) top = __vmaxu2(top, w[i] & 0x7fff7fffu);
        top = max(top << 16, top & 0xffff0000u);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, w[i] & 0x7fffffffu);
      }
      const bool mine = in(j * a.step);
      if (top >= 0x7f800000u) {                    // an infinity or NaN
        top = 0;
#pragma unroll
        for (int i = 0; i < C; ++i) {
          f[i] = f[i] != f[i] ? 0.f : fminf(fmaxf(f[i], -3.4e38f), 3.4e38f);
          top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
        }
        if (mine) code = max(code, (int)BRISK_ERR_NUMERIC);
      }
#pragma unroll
      for (int o = 1; o < LANES; o <<= 1) top = max(top, __shfl_xor_sync(FULL_MASK, top, o));
      const uint32_t byte = scale_byte<T>(__uint_as_float(top));
      const uint32_t put = codes_of<T>(f, scale_value(byte));
      if (!mine) continue;
      uint8_t* p = codes + (unsigned long long)(uint32_t)(j * a.step) * to.tok;
      if constexpr (C == 8) *reinterpret_cast<uint32_t*>(p) = put;
      else *reinterpret_cast<uint16_t*>(p) = (uint16_t)put;
      if (at.c % GROUP == 0) scales[(unsigned long long)(uint32_t)(j * a.step) * to.stok] = (uint8_t)byte;
    }
  }
  if (a.alone) {
    code = __syncthreads_or(code == BRISK_ERR_NUMERIC) ? BRISK_ERR_NUMERIC : (bad ? BRISK_ERR_INVALID_ARG : BRISK_OK);
    if (threadIdx.x == 0) *a.status = code;
  } else if (code != BRISK_OK) {
    atomicMax(a.status, code);                     // (cleared before; the largest, whatever the order)
  }
}

template <typename T, int EACH>
__global__ void __launch_bounds__(MOVE_THREADS) load_kernel(const __grid_constant__ PackedMoveArgs a) {
  constexpr int C = channels<T>();
  const int b = blockIdx.y;
  int start;
  bool bad;
  const int n = rows_of(a, b, &start, &bad);
  if (blockIdx.x == 0 && b == 0 && blockIdx.z == 0) {      // the call's status: rows asked for that no cache has
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
  const Place<T, EACH> at(a);
  if (!at.there) return;
  const Inside in(a, start, n, true, at.t);
  const long long first = start + (long long)at.t;
  uint32_t codes[2][EACH], byte[2][EACH];
#pragma unroll
  for (int value = 0; value < 2; ++value) {
    const PackedView& from = value ? a.vp : a.kp;
    const uint8_t* p = from.codes + b * from.seq + at.h * from.head + at.c / 2 + first * from.tok;
    const uint8_t* s = from.scales + b * from.sseq + at.h * from.shead + at.c / GROUP + first * from.stok;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      codes[value][j] = byte[value][j] = 0;
      if (in(j * a.step)) {
        const uint8_t* q = p + (unsigned long long)(uint32_t)(j * a.step) * from.tok;
        if constexpr (C == 8) codes[value][j] = __ldg(reinterpret_cast<const uint32_t*>(q));
        else codes[value][j] = __ldg(reinterpret_cast<const uint16_t*>(q));
        byte[value][j] = __ldg(s + (unsigned long long)(uint32_t)(j * a.step) * from.stok);
      }
    }
  }
#pragma unroll
  for (int value = 0; value < 2; ++value) {
    const CacheView& out = value ? a.v : a.k;
    char* to = const_cast<char*>(row_at(out, sizeof(T), b, at.h, at.c, at.t));
    const long long step = a.step * out.tok * (long long)sizeof(T);
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      if (at.t + j * a.step >= a.T) break;
      uint32_t x[4];
      from_codes(codes[value][j], x);
      const uint32_t s = scale_f16(byte[value][j]);
      float f[C];
#pragma unroll
      for (int i = 0; i < C / 2; ++i) {            // (the products are exact, in fp16 and in T)
        const uint32_t y = mul_f16(x[i], s);
        const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&y));
        f[2 * i] = z.x;
        f[2 * i + 1] = z.y;
      }
      if constexpr (C == 4) {
        __stcs(reinterpret_cast<float4*>(to + j * step), make_float4(f[0], f[1], f[2], f[3]));
      } else {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const __nv_bfloat162 y = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
          w[k] = *reinterpret_cast<const uint32_t*>(&y);
        }
        __stcs(reinterpret_cast<uint4*>(to + j * step), make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
  }
}

dim3 grid_of(const PackedMoveArgs& a, int each) {
  const int n = a.step * each;
  return dim3((unsigned)((a.T + n - 1) / n), a.B, (unsigned)((a.by_token.d + MOVE_THREADS - 1) / MOVE_THREADS));
}
// Tokens of a thread: one while its CTAs are few, as calls' latency goes (32 rows of 8 sequences written and read back,
// 8 heads of 128: one 8.2 us, two 9.4, four 12.4), then two, and four of calls that write many (64 times 512 rows
// written: two 37.1 us, four 31.7; 16 prompts of 1500 to 4096: two 49.5, four 43.9; 64 caches read back: one 130,
// two 105, four 109).
int tokens_each(const PackedMoveArgs& a, bool writes) {
  auto ctas = [&](int each) {
    const dim3 g = grid_of(a, each);
    return (long long)g.x * g.y * g.z;
  };
  if (ctas(1) <= 4 * CACHE_SMS) return 1;
  return writes && ctas(4) >= 8 * CACHE_SMS ? 4 : 2;
}
template <typename T>
cudaError_t store(const PackedMoveArgs& a, dim3 grid, int each, cudaStream_t stream) {
  if (each == 1) store_kernel<T, 1><<<grid, MOVE_THREADS, 0, stream>>>(a);
  else if (each == 2) store_kernel<T, 2><<<grid, MOVE_THREADS, 0, stream>>>(a);
  else store_kernel<T, 4><<<grid, MOVE_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}
template <typename T>
cudaError_t load(const PackedMoveArgs& a, dim3 grid, int each, cudaStream_t stream) {
  if (each == 1) load_kernel<T, 1><<<grid, MOVE_THREADS, 0, stream>>>(a);
  else load_kernel<T, 2><<<grid, MOVE_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_packed_store(const PackedMoveArgs& args, cudaStream_t stream) {
  PackedMoveArgs a = args;
  const int each = tokens_each(a, true);
  const dim3 grid = grid_of(a, each);
  a.alone = grid.x == 1 && grid.y == 1 && grid.z == 1;
  cudaError_t e = a.alone ? cudaSuccess : cudaMemsetAsync(a.status, 0, sizeof(int32_t), stream);
  if (e != cudaSuccess) return e;
  return a.dt == BRISK_DT_BF16 ? store<__nv_bfloat16>(a, grid, each, stream) : store<float>(a, grid, each, stream);
}

cudaError_t launch_packed_load(const PackedMoveArgs& a, cudaStream_t stream) {
  const int each = tokens_each(a, false);
  const dim3 grid = grid_of(a, each);
  return a.dt == BRISK_DT_BF16 ? load<__nv_bfloat16>(a, grid, each, stream) : load<float>(a, grid, each, stream);
}

}  // namespace brisk
