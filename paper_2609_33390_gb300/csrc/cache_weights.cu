// Attention weight that each entry of the own caches got from a block's queries:
//
//   acc_out[b, h, t] = decay acc_in[b, h, t] + sum over the rows that see t of exp(scale q . k_t - lse)
//
// with the rows' log-sums lse that attention left. The keys are the tile's rows here: a key's sum
// over the query rows stays with its threads, so there are no atomics and the sums' order is fixed.
#include "cache.cuh"

namespace brisk {
namespace {

constexpr int W_THREADS = 256;
constexpr int W_KEYS = 64, W_ROWS = 64;
constexpr int WS = CACHE_MAX_D + 4;

template <typename T>
__global__ void __launch_bounds__(W_THREADS)
weights_simt_kernel(const __grid_constant__ WeightArgs a) {
  extern __shared__ __align__(16) float smem[];
  float* sK = smem;                        // [W_KEYS][WS]
  float* sQ = sK + W_KEYS * WS;            // [W_ROWS][CACHE_MAX_D]
  float* sL = sQ + W_ROWS * CACHE_MAX_D;   // [W_ROWS] log-sums in log2 units
  int* sLim = reinterpret_cast<int*>(sL + W_ROWS);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int tiles = (a.S + W_KEYS - 1) / W_KEYS, D = a.D, nv = D / 4;
  const long long item = blockIdx.x / tiles;
  const int t0 = (int)(blockIdx.x % tiles) * W_KEYS, b = (int)(item / a.Hkv), h = (int)(item % a.Hkv);
  const int raw = a.own_len[b], len = min(max(raw, 0), a.S);
  if (raw != len && tid == 0) set_status(a.status, BRISK_ERR_INVALID_ARG);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const int rows = a.L * a.G;
  if (t0 < len) {
    const T* kb = static_cast<const T*>(a.ko.p) + b * a.ko.seq + h * a.ko.head;
    for (int e = tid; e < W_KEYS * nv; e += W_THREADS) {
      const int r = e / nv, c = 4 * (e - r * nv);
      store4(sK + r * WS + c, t0 + r < len ? load4(kb + (t0 + r) * a.ko.tok + c) : make_float4(0.f, 0.f, 0.f, 0.f));
    }
    for (int r0 = 0; r0 < rows; r0 += W_ROWS) {
      __syncthreads();
      for (int e = tid; e < W_ROWS * nv; e += W_THREADS) {
        const int r = e / nv, c = 4 * (e - r * nv), i = (r0 + r) / a.G;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r0 + r < rows)
          v = load4(static_cast<const T*>(a.q.p) + b * a.q.seq + i * a.q.tok +
                    (h * a.G + (r0 + r - i * a.G)) * a.q.head + c);
        store4(sQ + r * CACHE_MAX_D + c, v);
      }
      if (tid < W_ROWS) {
        int lim = 0;
        float ls = 0.f;
        if (r0 + tid < rows) {
          const int i = (r0 + tid) / a.G, g = r0 + tid - i * a.G;
          const long long token = (long long)b * a.L + i;
          lim = a.visible ? min(len, a.visible[token]) : len;
          ls = a.lse[token * (a.Hkv * a.G) + h * a.G + g] * LOG2E;
          if (ls == -INFINITY) lim = 0;    // a row that saw nothing
        }
        sLim[tid] = lim;
        sL[tid] = ls;
      }
      __syncthreads();
      float s[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
      for (int d = 0; d < D; d += 4) {
        float4 q[4], k[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = load4(sQ + (ty * 4 + i) * CACHE_MAX_D + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = load4(sK + (tx + 16 * j) * WS + d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] = fmaf(q[i].x, k[j].x, s[i][j]);
            s[i][j] = fmaf(q[i].y, k[j].y, s[i][j]);
            s[i][j] = fmaf(q[i].z, k[j].z, s[i][j]);
            s[i][j] = fmaf(q[i].w, k[j].w, s[i][j]);
          }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int lim = sLim[ty * 4 + i];
        const float ls = sL[ty * 4 + i];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (t0 + tx + 16 * j < lim) sum[j] += ex2(s[i][j] * a.sl2 - ls);
      }
    }
  }
  __syncthreads();
  float* part = sQ;                        // [16][W_KEYS]
#pragma unroll
  for (int j = 0; j < 4; ++j) part[ty * W_KEYS + tx + 16 * j] = sum[j];
  __syncthreads();
  const int t = t0 + tid;
  if (tid < W_KEYS && t < a.S) {
    float w = 0.f;
#pragma unroll
    for (int y = 0; y < 16; ++y) w += part[y * W_KEYS + tid];
    const long long at = item * a.S + t;
    if (a.acc_in) w += a.decay * a.acc_in[at];
    a.acc_out[at] = t < len ? w : 0.f;
  }
}

}  // namespace

cudaError_t launch_weights_simt(const WeightArgs& a, cudaStream_t stream) {
  const size_t smem = sizeof(float) * (W_KEYS * WS + W_ROWS * CACHE_MAX_D + 2 * W_ROWS);
  const long long grid = (long long)a.B * a.Hkv * ((a.S + W_KEYS - 1) / W_KEYS);
  auto run = [&](auto kernel) {
    cudaError_t e = set_up_kernel(kernel, CARVEOUT_FULL_KB, smem);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)grid, W_THREADS, smem, stream>>>(a);
    return cudaGetLastError();
  };
  if (grid == 0) return cudaSuccess;
  return a.dt == BRISK_DT_BF16 ? run(weights_simt_kernel<__nv_bfloat16>) : run(weights_simt_kernel<float>);
}

}  // namespace brisk
