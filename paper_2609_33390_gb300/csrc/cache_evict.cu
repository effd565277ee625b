// Eviction from the own caches by accumulated attention weight. Of a sequence's n entries, a key
// head keeps the `recent` newest and, among the others, those of largest weight (ties to the lowest
// index) up to `keep` in all; what is kept moves to other buffers in its old order.
#include "cache.cuh"

namespace brisk {
namespace {

constexpr int SELECT_EACH = 4;           // neighbouring entries of a thread
constexpr int BINS = 2048;

// Order-preserving key of a weight: larger weights have larger keys, -0 equals 0, NaN is below all.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (isnan(w)) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive sum over the CTA's threads; *total gets the sum of all. `part` holds a word a warp.
template <int THREADS>
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
  int w = lane < THREADS / 32 ? part[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(FULL_MASK, w, o);
    if (lane >= o) w += y;
  }
  *total = __shfl_sync(FULL_MASK, w, 31);
  const int before = __shfl_sync(FULL_MASK, w, warp > 0 ? warp - 1 : 0);
  return x + (warp > 0 ? before : 0);
}

// One CTA a (sequence, key head): the smallest kept key by three passes over 11, 11 and 10 of its bits,
// then the kept indices in order. Bound by the barriers and the passes' latency (2048 entries
// 6 us): the weights, a hundredth of the entries' bytes, stay in L1 after the first pass.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
select_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ int hist[BINS], part[32];
  __shared__ uint32_t s_prefix;
  __shared__ int s_room;
  let_next_begin();
  const int b = blockIdx.x / a.Hkv, h = blockIdx.x - b * a.Hkv, tid = threadIdx.x;
  const int n = clamped_len(a, b);
  if (h == 0 && tid == 0) a.len_to[b] = min(n, a.keep);
  const float* acc = a.acc + (long long)blockIdx.x * a.S;
  float* acc_to = a.acc_to + (long long)blockIdx.x * a.keep;
  int32_t* kept = a.kept + (long long)blockIdx.x * a.keep;
  if (n <= a.keep) {
    for (int i = tid; i < a.keep; i += THREADS) {
      kept[i] = i < n ? i : -1;
      acc_to[i] = i < n ? acc[i] : 0.f;
    }
    return;
  }
  const int m = n - a.recent;              // entries that may go; n > keep, so m > room
  int room = a.keep - a.recent;            // how many of them stay
  // the key of the last one that stays, and how many of its equals do
  uint32_t prefix = 0, known = 0;          // known: the bits of it that are
  const bool some = room > 0;
  if (some)
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : BINS;
#pragma unroll
      for (int i = 0; i < BINS; i += THREADS) hist[i + tid] = 0;
      __syncthreads();
      for (int i = tid; i < m; i += THREADS) {
        const uint32_t k = weight_key(acc[i]);
        if ((k & known) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1);
      }
      __syncthreads();
      // bins from the largest: thread j holds EACH from bins - 1 - EACH j downwards
      constexpr int EACH = BINS / THREADS;
      const int top = bins - 1 - EACH * tid;
      int count[EACH], mine = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) mine += count[i] = top > 0 ? hist[top - i] : 0;
      int total;
      int before = block_scan<THREADS>(mine, part, &total) - mine;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if (before < room && before + count[i] >= room) {
          s_prefix = prefix | (uint32_t)(top - i) << shift;
          s_room = room - before;
        }
        before += count[i];
      }
      __syncthreads();
      prefix = s_prefix;
      room = s_room;
      known |= (uint32_t)(bins - 1) << shift;
      __syncthreads();
    }
  int done = 0, equal = 0;                 // entries above the last key (and newest) seen, and its equals
  for (int i0 = 0; i0 < n; i0 += THREADS * SELECT_EACH) {
    const int i = i0 + tid * SELECT_EACH;
    float w[SELECT_EACH];
    int is = 0, in = 0;                    // two bits an entry: stays, equals
#pragma unroll
    for (int j = 0; j < SELECT_EACH; ++j) {
      w[j] = i + j < n ? acc[i + j] : 0.f;
      const uint32_t k = weight_key(w[j]);
      const bool old = i + j < m;
      if (i + j < n && (!old || (some && k > prefix))) is |= 1 << j;
      if (old && some && k == prefix) in |= 1 << j;
    }
    // both counts in one scan (a block has less than 2^15 entries)
    int total;
    const int mine = __popc(is) | __popc(in) << 16;
    const int upto = block_scan<THREADS>(mine, part, &total) - mine;
    int above = done + (upto & 0xffff), ties = equal + (upto >> 16);
#pragma unroll
    for (int j = 0; j < SELECT_EACH; ++j) {
      const bool tie = in >> j & 1, stay = (is >> j & 1) || (tie && ties < room);
      if (stay) {
        const int at = above + min(ties, room);
        kept[at] = i + j;
        acc_to[at] = w[j];
      }
      above += is >> j & 1;
      ties += tie;
    }
    done += total & 0xffff;
    equal += total >> 16;
  }
}

// The kept rows of keys and values, 16 bytes a thread at a time; zeros where there is none. The pieces of a
// sequence's (place, head) rows lie as in the target's token-major order, so that writes are runs of whole
// tokens; a thread's loads, of four pieces of the keys and of the values, are all on their way at once. Bound
// by the rows' bytes, read and written once (128 sequences cut to 2048 entries, 8 heads of 128: 319 us, 6.7 TB/s).
constexpr int MOVE_THREADS = 256, MOVE_EACH = 4;
__global__ void __launch_bounds__(MOVE_THREADS)
move_kernel(const __grid_constant__ EvictArgs a, Divisor by_vec, Divisor by_heads) {
  __shared__ int bad;
  const int b = blockIdx.y, first = (int)blockIdx.x * MOVE_THREADS * MOVE_EACH + threadIdx.x;
  const int rows = a.keep * a.Hkv, es = a.dt == BRISK_DT_BF16 ? 2 : 4, step = 16 / es;
  const char *kf = static_cast<const char*>(a.k.p) + b * a.k.seq * es, *vf = static_cast<const char*>(a.v.p) + b * a.v.seq * es;
  char *kt = static_cast<char*>(const_cast<void*>(a.k_to.p)) + b * a.k_to.seq * es;
  char *vt = static_cast<char*>(const_cast<void*>(a.v_to.p)) + b * a.v_to.seq * es;
  if (blockIdx.x == 0 && b == 0) {         // the call's status: the lengths that were clamped
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.B; i += MOVE_THREADS)
      if (a.own_len[i] < 0 || a.own_len[i] > a.S) bad = 1;
    __syncthreads();
    if (threadIdx.x == 0) *a.status = bad ? BRISK_ERR_INVALID_ARG : BRISK_OK;
  }
  wait_for_previous();
  int h[MOVE_EACH], at[MOVE_EACH], c[MOVE_EACH], src[MOVE_EACH];
#pragma unroll
  for (int j = 0; j < MOVE_EACH; ++j) {
    const int e = first + j * MOVE_THREADS, row = by_vec.of(e);
    at[j] = by_heads.of(row);
    h[j] = row - at[j] * a.Hkv;
    c[j] = (e - row * by_vec.d) * step;
    // (select_kernel wrote it while this kernel was set up: no load that takes memory for unchanging)
    src[j] = row < rows ? a.kept[((long long)b * a.Hkv + h[j]) * a.keep + at[j]] : -2;
  }
  uint4 x[MOVE_EACH], y[MOVE_EACH];
#pragma unroll
  for (int j = 0; j < MOVE_EACH; ++j) {
    x[j] = y[j] = make_uint4(0, 0, 0, 0);
    if (src[j] >= 0) {
      x[j] = ld_stream_v4(kf + (src[j] * a.k.tok + h[j] * a.k.head + c[j]) * es);
      y[j] = ld_stream_v4(vf + (src[j] * a.v.tok + h[j] * a.v.head + c[j]) * es);
    }
  }
#pragma unroll
  for (int j = 0; j < MOVE_EACH; ++j)
    if (src[j] >= -1) {
      __stcs(reinterpret_cast<uint4*>(kt + (at[j] * a.k_to.tok + h[j] * a.k_to.head + c[j]) * es), x[j]);
      __stcs(reinterpret_cast<uint4*>(vt + (at[j] * a.v_to.tok + h[j] * a.v_to.head + c[j]) * es), y[j]);
    }
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, cudaStream_t stream) {
  const int es = a.dt == BRISK_DT_BF16 ? 2 : 4, nvec = a.D * es / 16;
  Divisor by_vec, by_heads;
  by_vec.set(nvec);
  by_heads.set(a.Hkv);
  // with more CTAs than two an SM, smaller ones, of which four fit (1024 selections of 1500 to 4096 entries: the call
  // 336 us, with the larger ones 342)
  const int ctas = a.B * a.Hkv;
  if (ctas > 2 * CACHE_SMS) select_kernel<512><<<ctas, 512, 0, stream>>>(a);
  else select_kernel<1024><<<ctas, 1024, 0, stream>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const long long vecs = (long long)a.keep * a.Hkv * nvec, each = MOVE_THREADS * MOVE_EACH;
  return launch_early(move_kernel, dim3((unsigned)((vecs + each - 1) / each), a.B), MOVE_THREADS, 0, stream, true, a, by_vec,
                      by_heads);
}

}  // namespace brisk
