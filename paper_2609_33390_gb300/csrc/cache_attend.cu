// Attention of a block's queries over a shared prefix and the sequences' own caches.
//
//   s_t = scale q . k_t,   lse = log sum_t exp(s_t),   out = sum_t exp(s_t - lse) v_t
//
// over the prefix's entries and the own entries that the query sees. A fragment (see Plan) keeps, for
// each of its rows, the running maximum m of its scores, l = sum exp(s - m) and O = sum exp(s - m) v;
// parts of one row join by l = sum_i l_i exp(m_i - m), O likewise, with m the largest of the m_i.
// Scores, sums and parts are fp32; maxima and scores are held in log2 units.
#include "cache.cuh"

namespace brisk {
namespace {

constexpr int SIMT_THREADS = 256;
constexpr int KT = ATTEND_KT_F32;
constexpr int KS = CACHE_MAX_D + 4;    // floats between the key tile's rows: 16 rows' float4s in two wavefronts

// Rows x keys on the FMA units: 16 x 16 threads, RT/16 rows and 4 keys each for the scores, the
// same rows and 8 columns each for the sums of values. A row's 16 threads are half a warp, so
// its maximum, its sum and the exchange of its probabilities need no barrier of the CTA.
template <typename T, int RT>
__global__ void __launch_bounds__(SIMT_THREADS)
attend_simt_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int RPT = RT / 16;
  extern __shared__ __align__(16) float smem[];
  float* sQ = smem;                               // [RT][CACHE_MAX_D]
  float* sK = sQ + RT * CACHE_MAX_D;              // [KT][KS]
  float* sV = sK + KT * KS;                       // [KT][CACHE_MAX_D]
  float* sP = sV + KT * CACHE_MAX_D;              // [RT][KT + 4]
  int32_t* cum = reinterpret_cast<int32_t*>(sP + RT * (KT + 4));
  __shared__ int warp_sum[SIMT_THREADS / 32], bad, lowest;

  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  if (tid == 0) bad = 0;
  __syncthreads();
  const int own = count_tiles<SIMT_THREADS>(a, KT, cum, warp_sum, &bad);
  const Plan plan(a, RT, KT, own);
  if (blockIdx.x == 0)
    for (int b = tid; b <= a.B; b += SIMT_THREADS) a.cum[b] = cum[b];
  if (tid == 0) a.errs[blockIdx.x] = bad && blockIdx.x == 0 ? BRISK_ERR_INVALID_ARG : BRISK_OK;

  const int D = a.D, nv = D / 4;
  Walk walk(plan, cum, blockIdx.x);
  Frag f;
  while (walk.next(plan, cum, f)) {
    const int len = f.prefix ? a.P : clamped_len(a, f.b);
    const T* kb = static_cast<const T*>(f.prefix ? a.kp.p : a.ko.p) +
                  (f.prefix ? f.h * a.kp.head : f.b * a.ko.seq + f.h * a.ko.head);
    const T* vb = static_cast<const T*>(f.prefix ? a.vp.p : a.vo.p) +
                  (f.prefix ? f.h * a.vp.head : f.b * a.vo.seq + f.h * a.vo.head);
    const long long ktok = f.prefix ? a.kp.tok : a.ko.tok, vtok = f.prefix ? a.vp.tok : a.vo.tok;
    __syncthreads();                               // the last fragment's reads are done
    if (tid == 0) lowest = len;
    for (int e = tid; e < RT * nv; e += SIMT_THREADS) {
      const int r = e / nv, c = 4 * (e - r * nv);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < f.rows) {
        int token, head;
        row_of(a, f, r, token, head);
        const int b = token / a.L, i = token - b * a.L;
        v = load4(static_cast<const T*>(a.q.p) + b * a.q.seq + i * a.q.tok + head * a.q.head + c);
      }
      store4(sQ + r * CACHE_MAX_D + c, v);
    }
    __syncthreads();
    int lim[RPT];
    float m[RPT], l[RPT], o[RPT][8];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int r = ty * RPT + i;
      lim[i] = 0;
      if (r < f.rows) {
        int token, head;
        row_of(a, f, r, token, head);
        lim[i] = row_limit(a, f, token, len);
        if (tx == 0 && lim[i] < len) atomicMin(&lowest, lim[i]);
      }
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[i][j] = 0.f;
    }
    __syncthreads();
    const int low = lowest;                        // entries from here on are hidden from some row

    for (int kt = f.k0; kt < f.k0 + f.n; ++kt) {
      const int t0 = kt * KT;
      bool odd = false;                            // an infinity or NaN that some row must not see
      for (int e = tid; e < KT * nv; e += SIMT_THREADS) {
        const int r = e / nv, c = 4 * (e - r * nv), t = t0 + r;
        float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
        if (t < len) {
          k = load4(kb + t * ktok + c);
          v = load4(vb + t * vtok + c);
          if (t >= low) odd |= !(isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w));
        }
        store4(sK + r * KS + c, k);
        store4(sV + r * CACHE_MAX_D + c, v);
      }
      odd = __syncthreads_or(odd);

      float s[RPT][4];
#pragma unroll
      for (int i = 0; i < RPT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
      for (int d = 0; d < D; d += 4) {
        float4 q[RPT], k[4];
#pragma unroll
        for (int i = 0; i < RPT; ++i) q[i] = load4(sQ + (ty * RPT + i) * CACHE_MAX_D + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = load4(sK + (tx + 16 * j) * KS + d);
#pragma unroll
        for (int i = 0; i < RPT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] = fmaf(q[i].x, k[j].x, s[i][j]);
            s[i][j] = fmaf(q[i].y, k[j].y, s[i][j]);
            s[i][j] = fmaf(q[i].z, k[j].z, s[i][j]);
            s[i][j] = fmaf(q[i].w, k[j].w, s[i][j]);
          }
      }
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[i][j] = t0 + tx + 16 * j < lim[i] ? s[i][j] * a.sl2 : -INFINITY;
          top = fmaxf(top, s[i][j]);
        }
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, x));
        const float mn = fmaxf(m[i], top), ms = mn == -INFINITY ? 0.f : mn;
        const float alpha = ex2(m[i] - ms);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = ex2(s[i][j] - ms);
          sum += p;
          sP[(ty * RPT + i) * (KT + 4) + tx + 16 * j] = p;
        }
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) sum += __shfl_xor_sync(FULL_MASK, sum, x);
        l[i] = l[i] * alpha + sum;
        m[i] = mn;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[i][j] *= alpha;
      }
      __syncwarp();
      const int c0 = 4 * tx, c1 = 64 + 4 * tx;
      if (!odd) {
#pragma unroll 4
        for (int t = 0; t < KT; ++t) {
          const float4 v0 = load4(sV + t * CACHE_MAX_D + c0), v1 = load4(sV + t * CACHE_MAX_D + c1);
#pragma unroll
          for (int i = 0; i < RPT; ++i) {
            const float p = sP[(ty * RPT + i) * (KT + 4) + t];
            o[i][0] = fmaf(p, v0.x, o[i][0]);
            o[i][1] = fmaf(p, v0.y, o[i][1]);
            o[i][2] = fmaf(p, v0.z, o[i][2]);
            o[i][3] = fmaf(p, v0.w, o[i][3]);
            o[i][4] = fmaf(p, v1.x, o[i][4]);
            o[i][5] = fmaf(p, v1.y, o[i][5]);
            o[i][6] = fmaf(p, v1.z, o[i][6]);
            o[i][7] = fmaf(p, v1.w, o[i][7]);
          }
        }
      } else {
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int i = 0; i < RPT; ++i) {
            const float p = sP[(ty * RPT + i) * (KT + 4) + t];
            if (t0 + t >= lim[i]) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              o[i][j] = fmaf(p, sV[t * CACHE_MAX_D + c0 + j], o[i][j]);
              o[i][4 + j] = fmaf(p, sV[t * CACHE_MAX_D + c1 + j], o[i][4 + j]);
            }
          }
      }
      __syncthreads();
    }

#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int r = ty * RPT + i;
      if (r >= f.rows) continue;
      int token, head;
      row_of(a, f, r, token, head);
      if (f.whole) {
        const bool none = row_idle(a, token) || l[i] == 0.f;
        const float inv = none ? 0.f : 1.f / l[i];
        T* to = static_cast<T*>(a.out) + ((long long)token * (a.Hkv * a.G) + head) * D;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int c = 64 * j + 4 * tx;
          if (c >= D) continue;
          store4(to + c, none ? make_float4(0.f, 0.f, 0.f, 0.f)
                              : make_float4(o[i][4 * j] * inv, o[i][4 * j + 1] * inv, o[i][4 * j + 2] * inv,
                                            o[i][4 * j + 3] * inv));
        }
        if (a.lse && tx == 0)
          a.lse[(long long)token * (a.Hkv * a.G) + head] = none ? -INFINITY : (m[i] + log2f(l[i])) * (1.f / LOG2E);
      } else {
        const int per = f.prefix ? min(RT, plan.R) : min(RT, plan.LG);
        const long long at = f.slot * per + r;
        float* to = (f.prefix ? a.part_p : a.part_o) + at * D;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int c = 64 * j + 4 * tx;
          if (c < D) store4(to + c, make_float4(o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]));
        }
        if (tx == 0) (f.prefix ? a.ml_p : a.ml_o)[at] = make_float2(m[i], l[i]);
      }
    }
  }
}

constexpr size_t simt_smem(int rt) {
  return sizeof(float) * (rt * CACHE_MAX_D + KT * KS + KT * CACHE_MAX_D + rt * (KT + 4)) +
         sizeof(int32_t) * (CACHE_MAX_B + 1);
}

// Joins the parts of the rows whose keys were divided: one warp a row, a lane four columns.
constexpr int MERGE_THREADS = 256;
template <typename T>
__global__ void __launch_bounds__(MERGE_THREADS)
merge_kernel(const __grid_constant__ AttendArgs a, int rt, int kt) {
  const int lane = threadIdx.x & 31;
  const Plan plan(a, rt, kt, a.cum[a.B]);
  const int Hq = a.Hkv * a.G;
  const int rows = a.B * a.L * Hq, per_p = min(rt, plan.R), per_o = min(rt, plan.LG);
  for (int row = (int)blockIdx.x * (MERGE_THREADS / 32) + (threadIdx.x >> 5); row < rows;
       row += (int)gridDim.x * (MERGE_THREADS / 32)) {
    const int token = row / Hq, head = row - token * Hq, h = head / a.G, g = head - h * a.G;
    const int b = token / a.L;
    // the parts over the prefix, then those over the own cache: a run of slots each
    long long at_p = 0, at_o = 0;
    int np = 0, no = 0;
    bool written = false;                           // by the only CTA that had these rows' keys
    if (plan.kP > 0) {
      const int r = token * a.G + g, pt = r / rt;
      const long long item = h * plan.nPT + pt;
      const int c0 = plan.cta_of(item * plan.kP), c1 = plan.cta_of(item * plan.kP + plan.kP - 1);
      np = c1 - c0 + 1;
      at_p = (item + c0) * per_p + (r - pt * rt);
      const int b0 = pt * rt / plan.LG, b1 = min(pt * rt + rt, plan.R) - 1;
      written = np == 1 && a.cum[b1 / plan.LG + 1] == a.cum[b0];
    }
    const int n = a.cum[b + 1] - a.cum[b];
    if (n > 0) {
      const int r = (token - b * a.L) * a.G + g, lt = r / rt;
      const long long u = plan.own_start(a.cum, b, h, lt);
      const int c0 = plan.cta_of(u), c1 = plan.cta_of(u + n - 1);
      no = c1 - c0 + 1;
      at_o = (((long long)b * a.Hkv + h) * plan.nLT + lt + c0) * per_o + (r - lt * rt);
    }
    if (written || (np == 0 && no == 1)) continue;
    float top = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!row_idle(a, token))
      for (int i0 = 0; i0 < np + no; i0 += 32) {
        const int i = i0 + lane;
        float2 ml = make_float2(-INFINITY, 0.f);
        if (i < np) ml = a.ml_p[at_p + i * per_p];
        else if (i < np + no) ml = a.ml_o[at_o + (i - np) * per_o];
        const float mn = fmaxf(top, warp_max(ml.x));
        const float ms = mn == -INFINITY ? 0.f : mn;
        const float w = ex2(ml.x - ms), was = ex2(top - ms);
        l = l * was + warp_sum((ml.x == mn ? 1.f : w) * ml.y);   // (a part without a finite score: 0, or NaN)
        o.x *= was; o.y *= was; o.z *= was; o.w *= was;
        top = mn;
        const int cnt = min(32, np + no - i0);
#pragma unroll 4
        for (int j = 0; j < cnt; ++j) {
          const float wj = __shfl_sync(FULL_MASK, w, j);
          const int k = i0 + j;
          const float* src = k < np ? a.part_p + (at_p + k * per_p) * a.D : a.part_o + (at_o + (k - np) * per_o) * a.D;
          if (4 * lane < a.D && wj != 0.f) {
            const float4 x = load4(src + 4 * lane);
            o.x = fmaf(wj, x.x, o.x);
            o.y = fmaf(wj, x.y, o.y);
            o.z = fmaf(wj, x.z, o.z);
            o.w = fmaf(wj, x.w, o.w);
          }
        }
      }
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    if (4 * lane < a.D)
      store4(static_cast<T*>(a.out) + (long long)row * a.D + 4 * lane, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    if (a.lse && lane == 0) a.lse[row] = none ? -INFINITY : (top + log2f(l)) * (1.f / LOG2E);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    int code = BRISK_OK;
    for (int c = 0; c < a.grid && code == BRISK_OK; ++c) code = a.errs[c];
    *a.status = code;
  }
}

}  // namespace

cudaError_t launch_attend_f32(const AttendArgs& a, cudaStream_t stream) {
  auto run = [&](auto kernel, size_t smem) {
    cudaError_t e = set_up_kernel(kernel, CARVEOUT_FULL_KB, smem);
    if (e != cudaSuccess) return e;
    kernel<<<a.grid, SIMT_THREADS, smem, stream>>>(a);
    return cudaGetLastError();
  };
  return run(attend_simt_kernel<float, ATTEND_RT_F32>, simt_smem(ATTEND_RT_F32));
}

cudaError_t launch_merge(const AttendArgs& a, cudaStream_t stream) {
  const int rows = a.B * a.L * a.Hkv * a.G, ctas = (rows + MERGE_THREADS / 32 - 1) / (MERGE_THREADS / 32);
  const int grid = ctas < 8 * CACHE_SMS ? ctas : 8 * CACHE_SMS;
  if (a.dt == BRISK_DT_BF16)
    merge_kernel<__nv_bfloat16><<<grid, MERGE_THREADS, 0, stream>>>(a, attend_rt(a.dt), attend_kt(a.dt));
  else
    merge_kernel<float><<<grid, MERGE_THREADS, 0, stream>>>(a, attend_rt(a.dt), attend_kt(a.dt));
  return cudaGetLastError();
}

}  // namespace brisk
