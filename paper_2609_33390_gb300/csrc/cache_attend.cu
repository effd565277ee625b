// Attention of a block's queries over a shared prefix and the sequences' own caches.
//
//   s_t = scale q . k_t,   lse = log sum_t exp(s_t),   out = sum_t exp(s_t - lse) v_t
//
// over the prefix's entries and the own entries that the query sees. A fragment (see Plan) keeps, for
// each of its rows, the running maximum m of its scores, l = sum exp(s - m) and O = sum exp(s - m) v;
// parts of one row join by l = sum_i l_i exp(m_i - m), O likewise, with m the largest of the m_i.
// Scores, sums and parts are fp32; maxima and scores are held in log2 units.
#include <type_traits>

#include "cache.cuh"
#include "tensor_core.cuh"

namespace brisk {
namespace {

constexpr int SIMT_THREADS = 256;
constexpr int KT = SIMT_KT, RT = SIMT_ROWS;
constexpr int KS = CACHE_MAX_D + 4;    // floats between the key tile's rows: 16 rows' float4s in two wavefronts
constexpr int PS = KT + 4;

// fp32: rows x keys on the FMA units. 16 x 16 threads, RPT rows and 4 keys each for the scores, the same rows
// and 8 columns each for the sums of values, two products an instruction. A row's 16 threads are half a warp, so
// its maximum, its sum and the exchange of its probabilities need no barrier of the CTA. RPT is 4, or 1
// where a fragment has at most 16 rows, for which the others would be padding (16 sequences of 16 rows: 226 us, with 4
// rows a thread 266). The probabilities lie over the keys, so that two CTAs fit an SM and one computes while the
// other's tile arrives. Bound by shared-memory reads and FMA issue, about evenly, with 64 rows (8 blocks of 64 positions,
// 32 heads on 8, D = 128, over 2000 + 200 to 500 entries: 545 us, 36 TFLOP/s); by shared-memory reads with few.
struct SimtTile {
  float *q, *k, *v;                    // [RT][CACHE_MAX_D], [KT][KS], [KT][CACHE_MAX_D]
};

__device__ __forceinline__ float4 fma4(float w, float4 x, float4 o) {
  return make_float4(fmaf(w, x.x, o.x), fmaf(w, x.y, o.y), fmaf(w, x.z, o.z), fmaf(w, x.w, o.w));
}
__device__ __forceinline__ float4 mul4(float w, float4 x) { return make_float4(w * x.x, w * x.y, w * x.z, w * x.w); }

// The end of a fragment's row whose sums are x, l and maximum m: its result where no other part exists, or a part.
struct RowEnd {
  float w;
  bool none;
  long long row;
  int per, r;
  __device__ RowEnd(const AttendArgs& a, const Frag& f, int r_, float m, float l) {
    int token, head;
    r = r_;
    row_of(a, f, r, token, head);
    row = (long long)token * (a.Hkv * a.G) + head;
    none = f.whole && (row_idle(a, token) || l == 0.f);
    w = !f.whole ? 1.f : (none ? 0.f : 1.f / l);
    per = min(RT, a.L * a.G * (f.prefix ? a.B : 1));
  }
  __device__ void store(const AttendArgs& a, const Frag& f, int c, float4 x) const {
    float* part = (f.prefix ? a.part_p : a.part_o) + part_at(f.slot, per, a.D, r, c);
    store4(f.whole ? static_cast<float*>(a.out) + row * a.D + c : part, none ? make_float4(0.f, 0.f, 0.f, 0.f) : mul4(w, x));
  }
  __device__ void store_sums(const AttendArgs& a, const Frag& f, float m, float l) const {
    if (!f.whole) (f.prefix ? a.ml_p : a.ml_o)[(long long)f.slot * per + r] = make_float2(m, l);
    else if (a.lse) a.lse[row] = none ? -INFINITY : (m + log2f(l)) * (1.f / LOG2E);
  }
};

template <int RPT>
__device__ __forceinline__ void simt_fragment(const AttendArgs& a, const Frag& f, const SimtTile& t,
                                              int* lowest) {
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, D = a.D, nv = D / 4, len = f.len;
  float* sP = t.k;                     // [RT][PS]
  const CacheView &kc = f.prefix ? a.kp : a.ko, &vc = f.prefix ? a.vp : a.vo;
  const float* kb = static_cast<const float*>(kc.p) + (f.prefix ? 0 : f.b * kc.seq) + f.h * kc.head;
  const float* vb = static_cast<const float*>(vc.p) + (f.prefix ? 0 : f.b * vc.seq) + f.h * vc.head;
  __syncthreads();                     // the last fragment's reads are done
  if (tid == 0) *lowest = len;
  for (int e = tid; e < RPT * 16 * nv; e += SIMT_THREADS) {
    const int r = e / nv, c = 4 * (e - r * nv);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < f.rows) {
      int token, head;
      row_of(a, f, r, token, head);
      const int b = a.by_L.of(token), i = token - b * a.L;
      v = load4(static_cast<const float*>(a.q.p) + b * a.q.seq + i * a.q.tok + head * a.q.head + c);
    }
    store4(t.q + r * CACHE_MAX_D + c, v);
  }
  __syncthreads();
  int lim[RPT];
  float m[RPT], l[RPT];
  f32x2 o[RPT][4];                     // columns 4 tx .. 4 tx + 3 and 64 more
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = ty * RPT + i;
    lim[i] = 0;
    if (r < f.rows) {
      int token, head;
      row_of(a, f, r, token, head);
      lim[i] = row_limit(a, f, token, len);
      if (tx == 0 && lim[i] < len) atomicMin(lowest, lim[i]);
    }
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[i][j] = pack2(0.f, 0.f);
  }
  __syncthreads();
  const int low = *lowest;             // entries from here on are hidden from some row

  for (int kt = f.k0; kt < f.k0 + f.n; ++kt) {
    const int t0 = kt * KT;
    copy_tile<KT, SIMT_THREADS>(t.k, KS, kb, kc.tok, t0, len, nv);
    asm volatile("cp.async.commit_group;" ::: "memory");
    copy_tile<KT, SIMT_THREADS>(t.v, CACHE_MAX_D, vb, vc.tok, t0, len, nv);
    asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 1;" ::: "memory");
    __syncthreads();

    f32x2 s2[RPT][4];                  // sums over the even and the odd columns
#pragma unroll
    for (int i = 0; i < RPT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s2[i][j] = pack2(0.f, 0.f);
#pragma unroll 2
    for (int d = 0; d < D; d += 4) {
      ulonglong2 q[RPT], k[4];
#pragma unroll
      for (int i = 0; i < RPT; ++i) q[i] = *reinterpret_cast<const ulonglong2*>(t.q + (ty * RPT + i) * CACHE_MAX_D + d);
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const ulonglong2*>(t.k + (tx + 16 * j) * KS + d);
#pragma unroll
      for (int i = 0; i < RPT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s2[i][j] = fma2(q[i].y, k[j].y, fma2(q[i].x, k[j].x, s2[i][j]));
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    bool odd = false;                  // an infinity or NaN that some row must not see
    if (t0 + KT > low)
      for (int e = tid; e < KT * nv; e += SIMT_THREADS) {
        const int r = e / nv;
        if (t0 + r < low) continue;
        const float4 v = load4(t.v + r * CACHE_MAX_D + 4 * (e - r * nv));
        odd |= !(isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w));
      }
    odd = __syncthreads_or(odd);       // the keys are read: the probabilities take their place
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      float s[4], top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x, y;
        unpack2(s2[i][j], x, y);
        s[j] = t0 + tx + 16 * j < lim[i] ? (x + y) * a.sl2 : -INFINITY;
        top = fmaxf(top, s[j]);
      }
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, x));
      const float mn = fmaxf(m[i], top), ms = mn == -INFINITY ? 0.f : mn, alpha = ex2(m[i] - ms);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = ex2(s[j] - ms);
        sum += p;
        sP[(ty * RPT + i) * PS + tx + 16 * j] = p;
      }
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) sum += __shfl_xor_sync(FULL_MASK, sum, x);
      l[i] = l[i] * alpha + sum;
      m[i] = mn;
      const f32x2 alpha2 = pack2(alpha, alpha);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = fma2(alpha2, o[i][j], pack2(0.f, 0.f));
    }
    __syncwarp();
    const int c0 = 4 * tx, c1 = 64 + 4 * tx;
    auto add_values = [&](auto wide) {             // (up to 64 columns: the first four of a thread)
#pragma unroll 2
      for (int y = 0; y < KT; y += 4) {
        float4 p[RPT];
#pragma unroll
        for (int i = 0; i < RPT; ++i) p[i] = load4(sP + (ty * RPT + i) * PS + y);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const ulonglong2 v0 = *reinterpret_cast<const ulonglong2*>(t.v + (y + e) * CACHE_MAX_D + c0);
          ulonglong2 v1;
          if (wide) v1 = *reinterpret_cast<const ulonglong2*>(t.v + (y + e) * CACHE_MAX_D + c1);
#pragma unroll
          for (int i = 0; i < RPT; ++i) {
            const float w = e == 0 ? p[i].x : (e == 1 ? p[i].y : (e == 2 ? p[i].z : p[i].w));
            const f32x2 w2 = pack2(w, w);
            o[i][0] = fma2(w2, v0.x, o[i][0]);
            o[i][1] = fma2(w2, v0.y, o[i][1]);
            if (wide) {
              o[i][2] = fma2(w2, v1.x, o[i][2]);
              o[i][3] = fma2(w2, v1.y, o[i][3]);
            }
          }
        }
      }
    };
    if (!odd) {
      if (D > 64) add_values(std::true_type{});
      else add_values(std::false_type{});
    } else {
      for (int y = 0; y < KT; ++y)
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
          if (t0 + y >= lim[i]) continue;
          const float w = sP[(ty * RPT + i) * PS + y];
          const f32x2 w2 = pack2(w, w);
          const ulonglong2 v0 = *reinterpret_cast<const ulonglong2*>(t.v + y * CACHE_MAX_D + c0);
          const ulonglong2 v1 = *reinterpret_cast<const ulonglong2*>(t.v + y * CACHE_MAX_D + c1);
          o[i][0] = fma2(w2, v0.x, o[i][0]);
          o[i][1] = fma2(w2, v0.y, o[i][1]);
          o[i][2] = fma2(w2, v1.x, o[i][2]);
          o[i][3] = fma2(w2, v1.y, o[i][3]);
        }
    }
    __syncthreads();
  }

#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = ty * RPT + i;
    if (r >= f.rows) continue;
    const RowEnd e(a, f, r, m[i], l[i]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = 64 * j + 4 * tx;
      if (c >= D) continue;
      float4 x;
      unpack2(o[i][2 * j], x.x, x.y);
      unpack2(o[i][2 * j + 1], x.z, x.w);
      e.store(a, f, c, x);
    }
    if (tx == 0) e.store_sums(a, f, m[i], l[i]);
  }
}

// fp32, a fragment of at most R <= 8 rows, as single tokens have them: a warp takes 8 keys at a time, its own
// running maximum, sums and O, and the warps' meet at the end. For the scores 4 lanes share a key, 16 bytes of it
// in turn; for the sums of values a lane has 4 columns, of every key or (up to 64 columns) of every other. Keys and
// values go through a ring of a warp's own, in which every lane reads what it copied itself: nobody waits for
// another, and two of the ring's three places are on their way (loads to registers go through what L1 shared memory
// leaves: 3.5 TB/s at most). Bound by the entries' bytes: 64 single tokens, 32 heads on 8, over 1000 to 2000 entries
// of 128 columns 143 us, 5.5 TB/s.
constexpr int FEW_KEYS = 8, SIMT_WARPS = SIMT_THREADS / 32, FEW_PLACES = 3;
constexpr int FEW_PIECES = FEW_KEYS * CACHE_MAX_D / 4 / 32;                  // 16 bytes each, a lane has of a place
template <int R>
struct FewShape {
  static constexpr int RING = SIMT_WARPS * FEW_PLACES * FEW_PIECES * 32 * 4; // floats
  static constexpr int O = SIMT_WARPS * R * CACHE_MAX_D;                     // (over the ring)
  static_assert(O <= RING, "");
  static constexpr int SMEM = 4 * (RING + R * CACHE_MAX_D + SIMT_WARPS * R * (FEW_KEYS + 2) + R);
};

template <int R>
__device__ __forceinline__ void few_fragment(const AttendArgs& a, const Frag& f, float* smem) {
  constexpr int PL = FEW_PIECES * 32 * 4;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, D = a.D, nv = D / 4;
  float* sO = smem;                                // [SIMT_WARPS][R][CACHE_MAX_D]
  float* ring = smem + warp * FEW_PLACES * PL + 4 * lane;                    // [place][piece][lane][4]
  float* sQ = smem + FewShape<R>::RING;            // [R][CACHE_MAX_D]
  float* sP = sQ + R * CACHE_MAX_D + warp * FEW_KEYS * R;                    // [FEW_KEYS][R] a warp
  float2* sM = reinterpret_cast<float2*>(sQ + R * CACHE_MAX_D + SIMT_WARPS * FEW_KEYS * R);   // [SIMT_WARPS][R]
  int* sLim = reinterpret_cast<int*>(sM + SIMT_WARPS * R);
  const CacheView &kc = f.prefix ? a.kp : a.ko, &vc = f.prefix ? a.vp : a.vo;
  const float* kb = static_cast<const float*>(kc.p) + (f.prefix ? 0 : f.b * kc.seq) + f.h * kc.head;
  const float* vb = static_cast<const float*>(vc.p) + (f.prefix ? 0 : f.b * vc.seq) + f.h * vc.head;
  const bool narrow = D <= 64;
  const int sub = narrow ? lane >> 4 : 0, vcol = 4 * (narrow ? lane & 15 : lane), each = narrow ? 2 : 1;
  const int end = min((f.k0 + f.n) * KT, f.len), first = f.k0 * KT + warp * FEW_KEYS;
  const int pieces = (D + 15) / 16;                // of a key that a lane has
  // load number 2 i: the keys of the warp's step i; 2 i + 1: its values; zeros beyond the end
  auto fetch = [&](int load) {
    const int t0 = first + (load >> 1) * (SIMT_WARPS * FEW_KEYS);
    const uint32_t to = su32(ring + load % FEW_PLACES * PL);
    if (t0 < end)
#pragma unroll
      for (int j = 0; j < FEW_PIECES; ++j) {
        const bool v = load & 1;
        const int key = v ? t0 + j * each + sub : t0 + (lane >> 2), c = v ? vcol : 4 * (4 * j + (lane & 3));
        if (v ? j * each >= FEW_KEYS : j >= pieces) break;
        const bool there = key < end && c < D;
        const float* from = v ? vb + key * vc.tok + c : kb + key * kc.tok + c;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + j * 512), "l"(there ? from : kb),
                     "r"(there ? 16 : 0)
                     : "memory");
      }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  __syncthreads();                                 // the last fragment's reads are done
  fetch(0);
  fetch(1);
  const int nq = 4 * pieces;                       // (columns that lanes without a piece of a key multiply by zeros)
  for (int e = tid; e < R * nq; e += SIMT_THREADS) {
    const int r = e / nq, c = 4 * (e - r * nq);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < f.rows && c < D) {
      int token, head;
      row_of(a, f, r, token, head);
      const int b = a.by_L.of(token), i = token - b * a.L;
      v = load4(static_cast<const float*>(a.q.p) + b * a.q.seq + i * a.q.tok + head * a.q.head + c);
    }
    store4(sQ + r * CACHE_MAX_D + c, v);
  }
  if (tid < R) {
    int token, head;
    row_of(a, f, min(tid, f.rows - 1), token, head);
    sLim[tid] = row_limit(a, f, token, f.len);     // (rows that are not there: as the last one)
  }
  __syncthreads();
  int low = f.len;                                 // entries from here on are hidden from some row
#pragma unroll
  for (int r = 0; r < R; ++r) low = min(low, sLim[r]);

  float m[R], l[R];                                // (l: of the lane's keys)
  f32x2 o[R][2];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
    o[r][0] = o[r][1] = pack2(0.f, 0.f);
  }
  int load = 0;
  for (int t0 = first; t0 < end; t0 += SIMT_WARPS * FEW_KEYS, load += 2) {
    fetch(load + 2);
    asm volatile("cp.async.wait_group 2;" ::: "memory");
    const float* k = ring + load % FEW_PLACES * PL;
    f32x2 x[R];
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = pack2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < FEW_PIECES; ++j) {
      if (j >= pieces) break;
      const ulonglong2 kj = *reinterpret_cast<const ulonglong2*>(k + j * 128);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(sQ + r * CACHE_MAX_D + 4 * (4 * j + (lane & 3)));
        x[r] = fma2(q.y, kj.y, fma2(q.x, kj.x, x[r]));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float s, top;
      unpack2(x[r], s, top);
      s += top;
      s += __shfl_xor_sync(FULL_MASK, s, 1);
      s += __shfl_xor_sync(FULL_MASK, s, 2);
      s = t0 + (lane >> 2) < sLim[r] ? s * a.sl2 : -INFINITY;
      top = s;
#pragma unroll
      for (int y = 4; y < 32; y <<= 1) top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, y));
      const float mn = fmaxf(m[r], top), ms = mn == -INFINITY ? 0.f : mn, alpha = ex2(m[r] - ms), p = ex2(s - ms);
      m[r] = mn;
      l[r] = l[r] * alpha + p;
      const f32x2 alpha2 = pack2(alpha, alpha);
      o[r][0] = fma2(alpha2, o[r][0], pack2(0.f, 0.f));
      o[r][1] = fma2(alpha2, o[r][1], pack2(0.f, 0.f));
      if ((lane & 3) == (r & 3)) sP[(lane >> 2) * R + r] = p;
    }
    __syncwarp();
    fetch(load + 3);
    asm volatile("cp.async.wait_group 2;" ::: "memory");
    const float* v = ring + (load + 1) % FEW_PLACES * PL;
    const bool hidden = t0 + FEW_KEYS > low;
#pragma unroll
    for (int y = 0; y < FEW_KEYS; ++y) {
      if (y * each >= FEW_KEYS) break;
      const int key = y * each + sub;
      const ulonglong2 vy = *reinterpret_cast<const ulonglong2*>(v + y * 128);
#pragma unroll
      for (int r = 0; r < R; r += 2) {
        const float2 w = *reinterpret_cast<const float2*>(sP + key * R + r);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          // (an infinity or NaN that the row must not see)
          if (hidden && t0 + key >= sLim[r + e]) continue;
          const f32x2 p2 = e ? pack2(w.y, w.y) : pack2(w.x, w.x);
          o[r + e][0] = fma2(p2, vy.x, o[r + e][0]);
          o[r + e][1] = fma2(p2, vy.y, o[r + e][1]);
        }
      }
    }
    __syncwarp();                                  // the probabilities are read
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();                                 // O's take the rings' place

#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) l[r] += __shfl_xor_sync(FULL_MASK, l[r], x);
    float4 x;
    unpack2(o[r][0], x.x, x.y);
    unpack2(o[r][1], x.z, x.w);
    if (narrow) {
      x.x += __shfl_xor_sync(FULL_MASK, x.x, 16);
      x.y += __shfl_xor_sync(FULL_MASK, x.y, 16);
      x.z += __shfl_xor_sync(FULL_MASK, x.z, 16);
      x.w += __shfl_xor_sync(FULL_MASK, x.w, 16);
    }
    if (vcol < D && sub == 0) store4(sO + (warp * R + r) * CACHE_MAX_D + vcol, x);
    if (lane == 0) sM[warp * R + r] = make_float2(m[r], l[r]);
  }
  __syncthreads();
  for (int e = tid; e < f.rows * nv; e += SIMT_THREADS) {
    const int r = e / nv, c = 4 * (e - r * nv);
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < SIMT_WARPS; ++w) top = fmaxf(top, sM[w * R + r].x);
    const float ms = top == -INFINITY ? 0.f : top;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < SIMT_WARPS; ++w) {
      const float2 ml = sM[w * R + r];
      const float wi = ml.x == top ? 1.f : ex2(ml.x - ms);
      sum += wi * ml.y;
      x = fma4(wi, load4(sO + (w * R + r) * CACHE_MAX_D + c), x);
    }
    const RowEnd end_of(a, f, r, top, sum);
    end_of.store(a, f, c, x);
    if (c == 0) end_of.store_sums(a, f, top, sum);
  }
}

// (FEW: rows a sequence has at most, where these are FEW_ROWS or less, else 0. One kernel for all forms would hold more
// code than the instruction cache.)
template <int FEW>
__global__ void __launch_bounds__(SIMT_THREADS, 2)
attend_simt_kernel(const __grid_constant__ AttendArgs a) {
  extern __shared__ __align__(16) float smem[];
  const SimtTile t{smem, smem + RT * CACHE_MAX_D, smem + RT * CACHE_MAX_D + KT * KS};
  __shared__ int warp_sum[SIMT_THREADS / 32], bad, lowest;
  __shared__ Start start;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  let_next_begin();
  const Plan own_plan =
      make_plan<SIMT_THREADS>(a, blockIdx.x, blockIdx.x == 0 ? a.cum : nullptr, warp_sum, &bad, &start);
  // (one thread walks through the units, in shared memory: the others need their registers)
  __shared__ Plan plan;
  __shared__ Walk walk;
  __shared__ Frag next;
  __shared__ int more;
  if (threadIdx.x == 0) {
    a.errs[blockIdx.x] = bad && blockIdx.x == 0 ? BRISK_ERR_INVALID_ARG : BRISK_OK;
    plan = own_plan;
    walk = Walk(a, plan, blockIdx.x, start);
  }
  for (;;) {
    if (threadIdx.x == 0) more = walk.next(a, plan, next);
    __syncthreads();
    if (!more) break;
    const Frag f = next;                           // (read before the fragment's first barrier)
    if constexpr (FEW > 0) {
      if (f.rows > FEW) simt_fragment<4>(a, f, t, &lowest);
      else few_fragment<FEW>(a, f, smem);
    } else {
      if (f.rows > 16) simt_fragment<4>(a, f, t, &lowest);
      else simt_fragment<1>(a, f, t, &lowest);
    }
  }
}

// The prefix alone, where own caches have a kernel of their own: parts, whatever its division.
__global__ void __launch_bounds__(SIMT_THREADS, 2)
attend_simt_prefix_kernel(const __grid_constant__ AttendArgs a) {
  extern __shared__ __align__(16) float smem[];
  const SimtTile t{smem, smem + RT * CACHE_MAX_D, smem + RT * CACHE_MAX_D + KT * KS};
  __shared__ int lowest;
  let_next_begin();
  const int R = a.B * a.L * a.G, kP = (a.P + KT - 1) / KT, nPT = (R + RT - 1) / RT, UP = a.Hkv * nPT * kP;
  const int2 range = units_of(blockIdx.x, max(1, (UP + a.sh.grid_p - 1) / a.sh.grid_p), UP);
  Frag f{};
  f.prefix = 1;
  f.len = a.P;
  for (int u = range.x; u < range.y; u += f.n) {
    const int item = u / kP;
    f.h = item / nPT;
    f.k0 = u - item * kP;
    f.n = min(kP - f.k0, range.y - u);
    f.row0 = (item - f.h * nPT) * RT;
    f.rows = min(RT, R - f.row0);
    f.slot = item + blockIdx.x;
    if (f.rows > 16) simt_fragment<4>(a, f, t, &lowest);
    else simt_fragment<1>(a, f, t, &lowest);
  }
  if (threadIdx.x == 0) a.errs[blockIdx.x] = BRISK_OK;
  wait_for_previous();                             // (the join waits for this kernel alone)
}

constexpr size_t SIMT_SMEM = sizeof(float) * (RT * CACHE_MAX_D + KT * KS + KT * CACHE_MAX_D);

// Joins the parts of the rows whose keys were divided.
//
// Many rows: a CTA takes 32 neighbouring rows of a key head, a row a lane and 16 columns a warp, so that loads
// are runs of 512 bytes as the parts lie; four parts' are on their way at once. Few rows: a CTA takes 4 rows, 8
// lanes each, and its 8 warps the rows' parts in turn, which meet in shared memory: one load after
// another is a latency each (one block of 32 positions over 4096 + 1100 entries, 21 parts a row: parts one by
// one 54 us). Either way the division of the work is looked up while the kernels before still run.
constexpr int MERGE_WARPS = 8, MERGE_THREADS = 32 * MERGE_WARPS;

struct Merge {                                     // what both forms know, in shared memory
  Divisor by_share_p, by_share_o;
  int warp_sum[MERGE_WARPS], bad;
  Start start;
};
__device__ __forceinline__ Plan begin_merge(const AttendArgs& a, int32_t* cum, Merge* k) {
  const Plan plan = make_plan<MERGE_THREADS>(a, -1, cum, k->warp_sum, &k->bad, &k->start);
  if (threadIdx.x == 0) k->by_share_p.set(plan.share_p);
  if (threadIdx.x == 32) k->by_share_o.set(plan.share_o);
  __syncthreads();
  return plan;
}
// Whether a kernel before has written a row with these parts.
__device__ __forceinline__ bool written(const AttendArgs& a, const Parts& pre, const Parts& own) {
  return a.sh.grid_p > 0 ? a.joins && pre.n == 1 && own.n <= JOIN_PARTS : (pre.n == 0 && own.n == 1) || (pre.n == 1 && a.S == 0);
}
__device__ __forceinline__ void merge_status(const AttendArgs& a) {
  if (blockIdx.x != 0 || threadIdx.x >= 32) return;
  int code = BRISK_OK;                             // the largest: a wait that gave up before a bad length
  for (int c = threadIdx.x; c < a.sh.grid_p + a.sh.grid_o; c += 32) code = max(code, a.errs[c]);
  code = __reduce_max_sync(FULL_MASK, code);
  if (threadIdx.x == 0) *a.status = code;
}
template <typename T>
__global__ void __launch_bounds__(MERGE_THREADS, 2)
merge_many_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int AHEAD = 4, COLS = 16;
  extern __shared__ int32_t cum[];                 // [B + 1] key tiles before each sequence
  __shared__ Merge known;
  const Plan plan = begin_merge(a, cum, &known);
  const int lane = threadIdx.x & 31, D = a.D, Hq = a.Hkv * a.G;
  // where the head is narrow, several groups of rows share the warps
  const int slices = (D + COLS - 1) / COLS, groups = MERGE_WARPS / slices;
  const int sub = (threadIdx.x >> 5) / slices, c0 = ((threadIdx.x >> 5) - sub * slices) * COLS;
  const int per_head = (plan.R + 31) / 32, all = per_head * a.Hkv;
  bool waited = false;
  for (int w = (int)blockIdx.x * groups + sub; w - sub < all; w += (int)gridDim.x * groups) {
    bool mine = w < all && sub < groups;           // (and not written by one of the kernels before)
    const int h = w / per_head, r = (w - h * per_head) * 32 + lane;
    mine = mine && r < plan.R;
    Parts pre{}, own{};                            // over the prefix, over the own entries
    int token = 0;
    if (mine) {
      token = a.by_G.of(r);
      pre = prefix_parts(a, plan, known.by_share_p, h, r);
      own = own_parts(a, plan, known.by_share_o, cum, h, r);
      if (written(a, pre, own)) mine = false;
    }
    if (!waited) wait_for_previous();
    waited = true;
    const bool idle = mine && row_idle(a, token);  // (used at the end: its load and the parts' go together)
    const int parts = mine ? pre.n + own.n : 0;
    float m = -INFINITY, l = 0.f;
    float4 o[COLS / 4];
#pragma unroll
    for (int k = 0; k < COLS / 4; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < parts; i0 += AHEAD) {
      float2 ml[AHEAD];
      float4 x[AHEAD][COLS / 4];
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) {
        const int i = min(i0 + e, parts - 1);
        const bool first = i < pre.n;
        const int per = first ? pre.per : own.per, at = (first ? i : i - pre.n) * per;
        const float* src = (first ? pre.sums : own.sums) + (long long)at * D;
        ml[e] = make_float2(-INFINITY, 0.f);
        if (i0 + e >= parts) continue;
        ml[e] = (first ? pre.ml : own.ml)[at];
#pragma unroll
        for (int k = 0; k < COLS / 4; ++k) x[e][k] = load4(src + min(c0 + 4 * k, D - 4) * per);
      }
      float mn = m;
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) mn = fmaxf(mn, ml[e].x);
      const float ms = mn == -INFINITY ? 0.f : mn;
      // (a part without a finite score has sums of 0, or NaN, which pass)
      const float was = m == mn ? 1.f : ex2(m - ms);
      m = mn;
      l *= was;
#pragma unroll
      for (int k = 0; k < COLS / 4; ++k) o[k] = mul4(was, o[k]);
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) {
        if (i0 + e >= parts) continue;
        const float wi = ml[e].x == mn ? 1.f : ex2(ml[e].x - ms);
        l += wi * ml[e].y;
#pragma unroll
        for (int k = 0; k < COLS / 4; ++k) o[k] = fma4(wi, x[e][k], o[k]);
      }
    }
    if (!mine) continue;
    const bool none = l == 0.f || idle;
    const float inv = none ? 0.f : 1.f / l;
    const long long row = (long long)token * Hq + h * a.G + (r - token * a.G);
    T* to = static_cast<T*>(a.out) + row * D;
#pragma unroll
    for (int k = 0; k < COLS / 4; ++k)
      if (c0 + 4 * k < D) store4(to + c0 + 4 * k, none ? make_float4(0.f, 0.f, 0.f, 0.f) : mul4(inv, o[k]));
    if (a.lse && c0 == 0) a.lse[row] = none ? -INFINITY : (m + log2f(l)) * (1.f / LOG2E);
  }
  if (!waited) wait_for_previous();
  merge_status(a);
}

template <typename T>
__global__ void __launch_bounds__(MERGE_THREADS, 3)
merge_few_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int NG = CACHE_MAX_D / 32, ROWS = 4;   // groups of four columns of a lane; rows of a CTA
  extern __shared__ int32_t cum[];                 // [B + 1] key tiles before each sequence
  __shared__ Merge known;
  __shared__ __align__(16) float sum_of[MERGE_WARPS][ROWS][CACHE_MAX_D + 4];
  __shared__ float2 ml_of[MERGE_WARPS][ROWS];
  const Plan plan = begin_merge(a, cum, &known);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = a.D, Hq = a.Hkv * a.G;
  const int groups = (plan.R + ROWS - 1) / ROWS;   // of a key head
  bool waited = false;
  for (int w = blockIdx.x; w < groups * a.Hkv; w += gridDim.x) {
    const int h = w / groups, r = (w - h * groups) * ROWS + (lane & 3), cq = lane >> 2;
    Parts pre{}, own{};
    bool mine = r < plan.R;
    int token = 0;
    if (mine) {
      token = a.by_G.of(r);
      pre = prefix_parts(a, plan, known.by_share_p, h, r);
      own = own_parts(a, plan, known.by_share_o, cum, h, r);
      if (written(a, pre, own)) mine = false;
    }
    if (!waited) wait_for_previous();
    waited = true;
    const bool idle = mine && row_idle(a, token);
    const int parts = mine ? pre.n + own.n : 0;
    float m = -INFINITY, l = 0.f;
    float4 o[NG];
#pragma unroll
    for (int k = 0; k < NG; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = warp; i0 < parts; i0 += 2 * MERGE_WARPS) {
      float2 ml[2];
      float4 x[2][NG];
#pragma unroll
      for (int e = 0; e < 2; ++e) {                // two parts' loads on their way at once
        const int i = min(i0 + e * MERGE_WARPS, parts - 1);
        const bool first = i < pre.n;
        const int per = first ? pre.per : own.per, at = (first ? i : i - pre.n) * per;
        const float* src = (first ? pre.sums : own.sums) + (long long)at * D;
        ml[e] = (first ? pre.ml : own.ml)[at];
        if (i0 + e * MERGE_WARPS >= parts) ml[e] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int k = 0; k < NG; ++k) {             // (columns beyond D: others again, not stored)
          const int c = 4 * cq + 32 * k;
          x[e][k] = load4(src + (c < D ? c : 0) * per);
        }
      }
      const float mn = fmaxf(m, fmaxf(ml[0].x, ml[1].x)), ms = mn == -INFINITY ? 0.f : mn;
      const float was = m == mn ? 1.f : ex2(m - ms);
      m = mn;
      l *= was;
#pragma unroll
      for (int k = 0; k < NG; ++k) o[k] = mul4(was, o[k]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (i0 + e * MERGE_WARPS >= parts) continue;
        const float wi = ml[e].x == mn ? 1.f : ex2(ml[e].x - ms);
        l += wi * ml[e].y;
#pragma unroll
        for (int k = 0; k < NG; ++k) o[k] = fma4(wi, x[e][k], o[k]);
      }
    }
    __syncthreads();                               // (the last rows' are read)
#pragma unroll
    for (int k = 0; k < NG; ++k)
      if (4 * cq + 32 * k < D) store4(&sum_of[warp][lane & 3][4 * cq + 32 * k], o[k]);
    if (cq == 0) ml_of[warp][lane & 3] = idle ? make_float2(-INFINITY, 0.f) : make_float2(m, l);
    __syncthreads();
    // warp j joins row j, a lane four columns
    const int rw = warp & 3;
    const long long row = (long long)token * Hq + h * a.G + (r - token * a.G);
    const bool row_mine = __shfl_sync(FULL_MASK, (int)mine, rw) != 0 && warp < ROWS;
    const long long to_row = __shfl_sync(FULL_MASK, row, rw);
    if (!row_mine) continue;
    float top = -INFINITY, all = 0.f;
#pragma unroll
    for (int j = 0; j < MERGE_WARPS; ++j) top = fmaxf(top, ml_of[j][rw].x);
    const float ms = top == -INFINITY ? 0.f : top;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int j = 0; j < MERGE_WARPS; ++j) {
      const float2 ml = ml_of[j][rw];
      const float wj = ml.x == top ? 1.f : ex2(ml.x - ms);
      all += wj * ml.y;
      if (4 * lane < D) v = fma4(wj, load4(&sum_of[j][rw][4 * lane]), v);
    }
    const bool none = all == 0.f;
    const float inv = none ? 0.f : 1.f / all;
    if (4 * lane < D)
      store4(static_cast<T*>(a.out) + to_row * D + 4 * lane, none ? make_float4(0.f, 0.f, 0.f, 0.f) : mul4(inv, v));
    if (a.lse && lane == 0) a.lse[to_row] = none ? -INFINITY : (top + log2f(all)) * (1.f / LOG2E);
  }
  if (!waited) wait_for_previous();
  merge_status(a);
}

}  // namespace

cudaError_t launch_attend_f32(const AttendArgs& a, cudaStream_t stream) {
  auto run = [&](auto kernel, size_t few_smem) {
    const size_t smem = few_smem > SIMT_SMEM ? few_smem : SIMT_SMEM;
    cudaError_t e = set_up_kernel(kernel, CARVEOUT_FULL_KB, smem);
    if (e != cudaSuccess) return e;
    kernel<<<a.sh.grid_o, SIMT_THREADS, smem, stream>>>(a);
    return cudaGetLastError();
  };
  const int rows = a.L * a.G;
  if (rows > FEW_ROWS) return run(attend_simt_kernel<0>, 0);
  if (rows > 4) return run(attend_simt_kernel<8>, FewShape<8>::SMEM);
  return rows > 2 ? run(attend_simt_kernel<4>, FewShape<4>::SMEM) : run(attend_simt_kernel<2>, FewShape<2>::SMEM);
}

cudaError_t launch_prefix_f32(const AttendArgs& a, cudaStream_t stream) {
  cudaError_t e = set_up_kernel(attend_simt_prefix_kernel, CARVEOUT_FULL_KB, SIMT_SMEM);
  return e != cudaSuccess ? e : launch_early(attend_simt_prefix_kernel, a.sh.grid_p, SIMT_THREADS, SIMT_SMEM, stream, true, a);
}

cudaError_t launch_merge(const AttendArgs& a, cudaStream_t stream) {
  // The form for few rows while its CTAs fit the chip at once or little more. Whole calls, few and many: 32 rows 11.3
  // and 12.0 us, 1024 rows (21 parts each) 23.5 and 29.4, 2048 76.4 and 74.1, 4096 39.3 and 37.7, 16384 78.5 and 63.9.
  const long long rows = (long long)a.B * a.L * a.G * a.Hkv;
  const bool few = rows <= 8 * CACHE_SMS;
  const long long ctas = few ? (long long)((a.B * a.L * a.G + 3) / 4) * a.Hkv : (long long)((a.B * a.L * a.G + 31) / 32) * a.Hkv;
  const int fit = (few ? 3 : 2) * CACHE_SMS, grid = (int)(ctas < fit ? ctas : fit);
  const size_t smem = sizeof(int32_t) * (a.B + 1);
  auto run = [&](auto kernel) {
    cudaError_t e = set_up_kernel(kernel, CARVEOUT_FULL_KB, smem);
    return e != cudaSuccess ? e : launch_early(kernel, grid, MERGE_THREADS, smem, stream, true, a);
  };
  if (a.dt == BRISK_DT_BF16) return few ? run(merge_few_kernel<__nv_bfloat16>) : run(merge_many_kernel<__nv_bfloat16>);
  return few ? run(merge_few_kernel<float>) : run(merge_many_kernel<float>);
}

}  // namespace brisk
