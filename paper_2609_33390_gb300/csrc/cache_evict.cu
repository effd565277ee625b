// Eviction from the own caches by accumulated attention weight. Of a sequence's n entries, a key
// head keeps the `recent` newest and, among the others, those of largest weight (ties to the lowest
// index) up to `keep` in all; what is kept moves to other buffers in its old order.
#include "cache.cuh"

namespace brisk {
namespace {

constexpr int SELECT_THREADS = 1024;

// Order-preserving key of a weight: larger weights have larger keys, -0 equals 0, NaN is below all.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (isnan(w)) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive sum over the CTA's threads; *total gets the sum of all. `part` holds a word a warp.
__device__ __forceinline__ int block_scan(int x, int* part, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(FULL_MASK, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                         // the last scan's words are read
  if (lane == 31) part[warp] = x;
  __syncthreads();
  int w = part[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(FULL_MASK, w, o);
    if (lane >= o) w += y;
  }
  *total = __shfl_sync(FULL_MASK, w, 31);
  const int before = __shfl_sync(FULL_MASK, w, warp > 0 ? warp - 1 : 0);
  return x + (warp > 0 ? before : 0);
}

// One CTA a (sequence, key head): the smallest kept key by four passes over 8 bits each, then the
// kept indices in order.
__global__ void __launch_bounds__(SELECT_THREADS)
select_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ int hist[256], part[32];
  __shared__ uint32_t s_prefix;
  __shared__ int s_room;
  const int b = blockIdx.x / a.Hkv, h = blockIdx.x - b * a.Hkv, tid = threadIdx.x;
  const int raw = a.own_len[b], n = min(max(raw, 0), a.S);
  if (raw != n && tid == 0) set_status(a.status, BRISK_ERR_INVALID_ARG);
  if (h == 0 && tid == 0) a.len_to[b] = min(n, a.keep);
  const float* acc = a.acc + (long long)blockIdx.x * a.S;
  float* acc_to = a.acc_to + (long long)blockIdx.x * a.keep;
  int32_t* kept = a.kept + (long long)blockIdx.x * a.keep;
  if (n <= a.keep) {
    for (int i = tid; i < a.keep; i += SELECT_THREADS) {
      kept[i] = i < n ? i : -1;
      acc_to[i] = i < n ? acc[i] : 0.f;
    }
    return;
  }
  const int m = n - a.recent;              // entries that may go; n > keep, so m > room
  int room = a.keep - a.recent;            // how many of them stay
  // the key of the last one that stays, and how many of its equals do
  uint32_t prefix = 0;
  if (room > 0)
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = tid; i < m; i += SELECT_THREADS) {
        const uint32_t k = weight_key(acc[i]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      // bins from the largest: thread j holds bin 255 - j
      const int mine = tid < 256 ? hist[255 - tid] : 0;
      int total;
      const int upto = block_scan(mine, part, &total);
      if (tid < 256 && upto >= room && upto - mine < room) {
        s_prefix = prefix | ((uint32_t)(255 - tid) << shift);
        s_room = room - (upto - mine);
      }
      __syncthreads();
      prefix = s_prefix;
      room = s_room;
      __syncthreads();
    }
  int done = 0, equal = 0;                 // entries kept, and equals of the last key seen, so far
  for (int i0 = 0; i0 < n; i0 += SELECT_THREADS) {
    const int i = i0 + tid;
    const float w = i < n ? acc[i] : 0.f;
    const uint32_t k = weight_key(w);
    const bool old = i < m, tie = old && room > 0 && k == prefix;
    int total;
    const int rank = block_scan(tie ? 1 : 0, part, &total);
    const bool stay = i < n && (!old || (a.keep > a.recent && k > prefix) || (tie && equal + rank <= room));
    equal += total;
    const int at = block_scan(stay ? 1 : 0, part, &total);
    if (stay) {
      kept[done + at - 1] = i;
      acc_to[done + at - 1] = w;
    }
    done += total;
  }
}

// The kept rows of keys and values, 16 bytes a thread at a time; zeros where there is none.
constexpr int MOVE_THREADS = 256, MOVE_EACH = 4;
__global__ void __launch_bounds__(MOVE_THREADS)
move_kernel(const __grid_constant__ EvictArgs a, int nvec, int es) {
  const long long per = (long long)a.B * a.keep * a.Hkv * nvec;
  const long long first = (long long)blockIdx.x * MOVE_THREADS * MOVE_EACH + threadIdx.x;
  const CacheView& from = blockIdx.y ? a.v : a.k;
  const CacheView& to = blockIdx.y ? a.v_to : a.k_to;
  const int ev = 16 / es;                  // elements of 16 bytes
  uint4 x[MOVE_EACH];
  char* dst[MOVE_EACH];
#pragma unroll
  for (int j = 0; j < MOVE_EACH; ++j) {
    const long long e = first + j * MOVE_THREADS;
    dst[j] = nullptr;
    x[j] = make_uint4(0, 0, 0, 0);
    if (e >= per) continue;
    const long long row = e / nvec;        // (sequence, place, head)
    const int c = (int)(e - row * nvec) * ev;
    const long long bj = row / a.Hkv;
    const int h = (int)(row - bj * a.Hkv), b = (int)(bj / a.keep), at = (int)(bj - (long long)b * a.keep);
    const int src = a.kept[((long long)b * a.Hkv + h) * a.keep + at];
    dst[j] = static_cast<char*>(const_cast<void*>(to.p)) + (b * to.seq + at * to.tok + h * to.head + c) * es;
    if (src >= 0)
      x[j] = *reinterpret_cast<const uint4*>(static_cast<const char*>(from.p) +
                                             (b * from.seq + src * from.tok + h * from.head + c) * es);
  }
#pragma unroll
  for (int j = 0; j < MOVE_EACH; ++j)
    if (dst[j]) *reinterpret_cast<uint4*>(dst[j]) = x[j];
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, cudaStream_t stream) {
  const int es = a.dt == BRISK_DT_BF16 ? 2 : 4, nvec = a.D * es / 16;
  select_kernel<<<a.B * a.Hkv, SELECT_THREADS, 0, stream>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const long long per = (long long)a.B * a.keep * a.Hkv * nvec, each = MOVE_THREADS * MOVE_EACH;
  move_kernel<<<dim3((unsigned)((per + each - 1) / each), 2), MOVE_THREADS, 0, stream>>>(a, nvec, es);
  return cudaGetLastError();
}

}  // namespace brisk
