// Attention over a shared prefix and own caches, the attention weight that own entries got, and the
// eviction by it: arguments, the division of attention's work over the SMs, and the join of its parts.
#pragma once

#include <cuda.h>

#include "brisk_internal.cuh"

namespace brisk {

constexpr int CACHE_MAX_B = 4096;    // sequences of a call (every CTA holds their tile counts)
constexpr int CACHE_MAX_D = 128;     // width of a head
constexpr int CACHE_SMS = 152;       // CTAs that share attention's work, at most

struct CacheView {   // element (s, t, h, :) at p + s*seq + t*tok + h*head, strides in elements
  const void* p;
  long long seq, tok, head;
};

struct AttendArgs {
  int B, L, G, Hkv, D, P, S;         // G query heads a key head
  int dt;                            // brisk_dtype of q, keys, values and out
  CacheView q, kp, vp, ko, vo;
  const int32_t* own_len;            // [B]
  const int32_t* visible;            // [B, L] or nullptr
  float sl2;                         // scale * log2(e)
  void* out;                         // [B, L, Hkv * G, D]
  float* lse;                        // [B, L, Hkv * G] or nullptr
  // workspace: parts of rows whose keys were divided, by slot (see Plan): sums (see part_at) and
  // (running maximum in log2 units, sum of exponentials)
  float *part_p, *part_o;
  float2 *ml_p, *ml_o;
  int32_t* cum;                      // [B + 1] key tiles of the sequences before each
  int32_t* errs;                     // [grid] what a CTA found wrong
  int32_t* status;
  int grid;
  long long wait_limit;
};

// ---------------------------------------------------------------- division of the work
// The unit of work is a tile of KT keys for a tile of up to RT query rows of one key head. A row is a
// (token, query head of the group) pair: row = token * G + g. Over the prefix, the rows of all
// sequences form common tiles (its keys are read once for RT rows, whichever sequence they are of);
// over the own caches, the rows of one sequence. All units stand in one sequence: first the prefix's
// (by head, row tile, key tile), then the own caches' (by sequence, head, row tile, key tile), and
// each CTA takes `share` of them, wherever that begins and ends. A row tile's keys may so
// be divided over several CTAs, each of which leaves a part; the parts are joined by merge_kernel.
// Slots: walking through the sequence, (item index + CTA) grows with every (item, CTA) pair, so it
// numbers the parts. Counts of units fit 31 bits (checked on the host).
struct Plan {
  int B, LG, Hkv, P, RT, KT;
  int nPT, kP, nLT;                  // row tiles and key tiles of the prefix; row tiles of a sequence
  int R, UP, T, share;               // rows a key head; units of the prefix; all units; units a CTA

  __device__ Plan(int b, int lg, int hkv, int p, int rt, int kt, int own_tiles, int grid) {
    B = b; LG = lg; Hkv = hkv; P = p; RT = rt; KT = kt;
    R = B * LG;
    kP = (P + KT - 1) / KT;
    nPT = P > 0 ? (R + RT - 1) / RT : 0;
    nLT = (LG + RT - 1) / RT;
    UP = Hkv * nPT * kP;
    T = UP + Hkv * nLT * own_tiles;
    share = max(1, (int)(((unsigned)T + grid - 1) / grid));
  }
  __device__ Plan(const AttendArgs& a, int rt, int kt, int own_tiles)
      : Plan(a.B, a.L * a.G, a.Hkv, a.P, rt, kt, own_tiles, a.grid) {}
  __device__ int units_of(int cta) const {
    return (int)(min((long long)T, (cta + 1LL) * share) - min((long long)T, (long long)cta * share));
  }
  __device__ int cta_of(int u) const { return u / share; }
  __device__ int own_start(const int32_t* cum, int b, int h, int lt) const {
    return UP + Hkv * nLT * cum[b] + (h * nLT + lt) * (cum[b + 1] - cum[b]);
  }
};

// A CTA's share of one item (a row tile's keys): key tiles [k0, k0 + n).
struct Frag {
  int prefix, whole;                 // whole: no other part for these rows exists
  int h, b, tile, k0, n;
  int row0, rows;                    // rows of the head over the prefix, of the sequence else
  int slot;
};

struct Walk {
  int u, end, c, b;

  __device__ Walk(const Plan& p, const int32_t* cum, int cta) {
    c = cta;
    b = 0;
    u = (int)min((long long)p.T, (long long)cta * p.share);
    end = (int)min((long long)p.T, (long long)u + p.share);
    if (end > p.UP) {                // the sequence of the first unit behind the prefix's
      const int v = (u > p.UP ? u - p.UP : 0) / (p.Hkv * p.nLT);
      int lo = 0, hi = p.B - 1;      // the last b with cum[b] <= v
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (cum[mid] <= v) lo = mid; else hi = mid - 1;
      }
      b = lo;
    }
  }
  __device__ bool next(const Plan& p, const int32_t* cum, Frag& f) {
    if (u >= end) return false;
    if (u < p.UP) {
      const int item = u / p.kP;
      f.prefix = 1;
      f.k0 = u - item * p.kP;
      f.n = min(p.kP - f.k0, end - u);
      f.h = item / p.nPT;
      f.tile = item - f.h * p.nPT;
      f.b = 0;
      f.row0 = f.tile * p.RT;
      f.rows = min(p.RT, p.R - f.row0);
      f.slot = item + c;
      const int b0 = f.row0 / p.LG, b1 = (f.row0 + f.rows - 1) / p.LG;
      f.whole = f.n == p.kP && cum[b1 + 1] == cum[b0];
    } else {
      const int per = p.Hkv * p.nLT;
      int base = p.UP + per * cum[b], n = cum[b + 1] - cum[b];
      while (u >= base + per * n) {
        base += per * n;
        ++b;
        n = cum[b + 1] - cum[b];
      }
      const int r = (u - base) / n;
      f.prefix = 0;
      f.b = b;
      f.h = r / p.nLT;
      f.tile = r - f.h * p.nLT;
      f.k0 = u - base - r * n;
      f.n = min(n - f.k0, end - u);
      f.row0 = f.tile * p.RT;
      f.rows = min(p.RT, p.LG - f.row0);
      f.slot = (b * p.Hkv + f.h) * p.nLT + f.tile + c;
      f.whole = f.n == n && p.P == 0;
    }
    u += f.n;
    return true;
  }
};

// A part's sums lie by groups of four columns, then rows: [D / 4][rows of a slot][4], so that neighbouring
// rows, which are neighbouring lanes of the kernels on both sides, lie side by side.
__device__ __forceinline__ long long part_at(long long slot, int per, int D, int row, int c) {
  return slot * per * D + ((long long)(c >> 2) * per + row) * 4;
}

template <typename Args>
__device__ __forceinline__ int clamped_len(const Args& a, int b) {
  return min(max(a.own_len[b], 0), a.S);
}
// Token (b * L + i) and query head of a fragment's row, and how many keys the row sees.
__device__ __forceinline__ void row_of(const AttendArgs& a, const Frag& f, int r, int& token, int& head) {
  const int row = f.row0 + r, t = row / a.G;
  head = f.h * a.G + (row - t * a.G);
  token = f.prefix ? t : f.b * a.L + t;
}
__device__ __forceinline__ int row_limit(const AttendArgs& a, const Frag& f, int token, int len) {
  if (f.prefix) return a.P;
  return a.visible ? max(0, min(len, a.visible[token])) : len;
}
__device__ __forceinline__ bool row_idle(const AttendArgs& a, int token) {
  return a.visible && a.visible[token] < 0;
}

// Key tiles before each sequence, by all THREADS threads of a CTA; returns their sum. *bad is set
// where a length lies outside 0..S (the caller clears it before a barrier).
template <int THREADS, typename Args>
__device__ int count_tiles(const Args& a, int kt, int32_t* cum, int* warp_sum, int* bad) {
  const int per = (a.B + THREADS - 1) / THREADS, tid = threadIdx.x, lane = tid & 31;
  const int b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
  int sum = 0;
  for (int b = b0; b < b1; ++b) {
    const int len = a.own_len[b];
    if (len < 0 || len > a.S) *bad = 1;
    sum += (min(max(len, 0), a.S) + kt - 1) / kt;
  }
  int run = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(FULL_MASK, run, o);
    if (lane >= o) run += x;
  }
  if (lane == 31) warp_sum[tid >> 5] = run;
  __syncthreads();
  int before = run - sum, total = 0;
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < (tid >> 5)) before += warp_sum[w];
    total += warp_sum[w];
  }
  for (int b = b0; b < b1; ++b) {
    cum[b] = before;
    before += (clamped_len(a, b) + kt - 1) / kt;
  }
  if (tid == 0) cum[a.B] = total;
  __syncthreads();
  return total;
}

// Four elements of a row, as fp32, and back.
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u),
                     __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v) {
  __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi));
}

// Rows and keys of a tile: bf16 on the tensor cores, fp32 on the FMA units.
constexpr int ATTEND_RT_TC = 256, ATTEND_KT_TC = 128;
constexpr int ATTEND_RT_F32 = 64, ATTEND_KT_F32 = 64;
inline int attend_rt(int dt) { return dt == BRISK_DT_BF16 ? ATTEND_RT_TC : ATTEND_RT_F32; }
inline int attend_kt(int dt) { return dt == BRISK_DT_BF16 ? ATTEND_KT_TC : ATTEND_KT_F32; }

// Tensor map of a cache's tiles of 64 columns x 128 entries (cache_attend_tc.cu).
bool make_cache_map(CUtensorMap* map, const CacheView& v, int D, int heads, int toks, int seqs);

cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t stream);
cudaError_t launch_attend_f32(const AttendArgs& a, cudaStream_t stream);
cudaError_t launch_merge(const AttendArgs& a, cudaStream_t stream);

// ---------------------------------------------------------------- attention weight of own entries
struct WeightArgs {
  int B, L, G, Hkv, D, S, dt;
  CacheView q, ko;
  const int32_t *own_len, *visible;
  const float* lse;        // [B, L, Hkv * G]
  float sl2, decay;
  const float* acc_in;     // [B, Hkv, S] or nullptr (zeros)
  float* acc_out;          // [B, Hkv, S]
  int32_t* status;
  int grid;
  long long wait_limit;
};
cudaError_t launch_weights_tc(const WeightArgs& a, cudaStream_t stream);
cudaError_t launch_weights_simt(const WeightArgs& a, cudaStream_t stream);

// ---------------------------------------------------------------- eviction
struct EvictArgs {
  int B, Hkv, D, S, dt, keep, recent;
  CacheView k, v, k_to, v_to;
  const float* acc;        // [B, Hkv, S]
  const int32_t* own_len;
  float* acc_to;           // [B, Hkv, keep]
  int32_t* len_to;         // [B]
  int32_t* kept;           // [B, Hkv, keep]
  int32_t* status;
};
cudaError_t launch_evict(const EvictArgs& a, cudaStream_t stream);

}  // namespace brisk
