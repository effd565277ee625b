// Attention weight that each entry of the own caches got from a block's queries:
//
//   acc_out[b, h, t] = decay acc_in[b, h, t] + sum over the rows that see t of exp(scale q . k_t - lse)
//
// with the rows' log-sums lse that attention left. The keys are the tile's rows here: a key's sum
// over the query rows stays with its threads, so there are no atomics and the sums' order is fixed.
// fp32 subtracts the log-sums as attention left them, in one fma with the scaled score, and takes the small difference
// to log2 units: with either of them in log2 units first, its rounding would be that of numbers the size of the
// scores, 4e-5 of a weight at scores of 500 (12 rows a head, 80 columns, scores of a few: error against 64 bits 1.0e-7,
// that way 3.3e-7).
#include <type_traits>

#include "cache.cuh"
#include "tensor_core.cuh"

namespace brisk {
namespace {

__device__ __forceinline__ float weight_of(float score, float scale, float lse) {
  return ex2(fmaf(score, scale, -lse) * LOG2E);
}

// fp32, more than FEW_W rows a head (see weights_few_kernel): tiles of 64 keys and 64 rows, 4 rows and 4 keys a thread. Bound by FMA issue and
// shared-memory reads (128 rows, 32 heads on 8, D = 128, 16 sequences of 1000 to 4000 entries: 326 us, 33 TFLOP/s).
constexpr int W_THREADS = 256;
constexpr int W_KEYS = 64, W_ROWS = 64;
constexpr int WS = CACHE_MAX_D + 4;

__global__ void __launch_bounds__(W_THREADS)
weights_simt_kernel(const __grid_constant__ WeightArgs a) {
  extern __shared__ __align__(16) float smem[];
  float* sK = smem;                        // [W_KEYS][WS]
  float* sQ = sK + W_KEYS * WS;            // [W_ROWS][CACHE_MAX_D]
  float* sL = sQ + W_ROWS * CACHE_MAX_D;   // [W_ROWS] log-sums
  int* sLim = reinterpret_cast<int*>(sL + W_ROWS);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int tiles = (a.S + W_KEYS - 1) / W_KEYS, D = a.D, nv = D / 4;
  const int item = blockIdx.x / tiles, t0 = (blockIdx.x - item * tiles) * W_KEYS, b = item / a.Hkv, h = item - b * a.Hkv;
  const int len = clamped_len(a, b);
  if (blockIdx.x == 0) {                   // the call's status: the lengths that were clamped
    bool bad = false;
    for (int i = tid; i < a.B; i += W_THREADS) bad |= a.own_len[i] < 0 || a.own_len[i] > a.S;
    bad = __syncthreads_or(bad);
    if (tid == 0) *a.status = bad ? BRISK_ERR_INVALID_ARG : BRISK_OK;
  }
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const int rows = a.L * a.G;
  if (t0 < len) {
    const float* kb = static_cast<const float*>(a.ko.p) + b * a.ko.seq + h * a.ko.head;
    copy_tile<W_KEYS, W_THREADS>(sK, WS, kb, a.ko.tok, t0, len, nv);
    for (int r0 = 0; r0 < rows; r0 += W_ROWS) {
      __syncthreads();
      for (int e = tid; e < (rows - r0 > 16 ? W_ROWS : 16) * nv; e += W_THREADS) {
        const int r = e / nv, c = 4 * (e - r * nv), row = min(r0 + r, rows - 1), i = a.by_G.of(row);
        copy16(sQ + r * CACHE_MAX_D + c, static_cast<const float*>(a.q.p) + b * a.q.seq + i * a.q.tok +
               (h * a.G + (row - i * a.G)) * a.q.head + c, r0 + r < rows);
      }
      if (tid < W_ROWS) {
        int lim = 0;
        float ls = 0.f;
        if (r0 + tid < rows) {
          const int i = a.by_G.of(r0 + tid), g = r0 + tid - i * a.G;
          const long long token = (long long)b * a.L + i;
          lim = a.visible ? min(len, a.visible[token]) : len;
          ls = a.lse[token * (a.Hkv * a.G) + h * a.G + g];
          if (ls == -INFINITY) lim = 0;    // a row that saw nothing
        }
        sLim[tid] = lim;
        sL[tid] = ls;
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncthreads();
      // 4 rows and 4 keys a thread, two products an instruction; a row where there are 16 at most
      auto add = [&](auto rows_each) {
        constexpr int RPT = decltype(rows_each)::value;
        f32x2 s2[RPT][4];                  // sums over the even and the odd columns
#pragma unroll
        for (int i = 0; i < RPT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s2[i][j] = pack2(0.f, 0.f);
#pragma unroll 2
        for (int d = 0; d < D; d += 4) {
          ulonglong2 q[RPT], k[4];
#pragma unroll
          for (int i = 0; i < RPT; ++i) q[i] = *reinterpret_cast<const ulonglong2*>(sQ + (ty * RPT + i) * CACHE_MAX_D + d);
#pragma unroll
          for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const ulonglong2*>(sK + (tx + 16 * j) * WS + d);
#pragma unroll
          for (int i = 0; i < RPT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s2[i][j] = fma2(q[i].y, k[j].y, fma2(q[i].x, k[j].x, s2[i][j]));
        }
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
          const int lim = sLim[ty * RPT + i];
          const float ls = sL[ty * RPT + i];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float x, y;
            unpack2(s2[i][j], x, y);
            if (t0 + tx + 16 * j < lim) sum[j] += weight_of(x + y, a.scale, ls);
          }
        }
      };
      if (rows - r0 > 16) add(std::integral_constant<int, 4>{});
      else add(std::integral_constant<int, 1>{});
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
    const long long at = (long long)item * a.S + t;
    if (a.acc_in) w += a.decay * a.acc_in[at];
    a.acc_out[at] = t < len ? w : 0.f;
  }
}

// fp32, up to FEW_W rows a head: a CTA has 128 keys, a warp 16, in registers: 4 lanes share a key, 16 bytes of it in
// turn, and a lane has a piece of two. A lane's 16 bytes of a query then serve both keys, and the lanes' sums of two
// rows and two keys are exchanged so that each has one pair's. Bound by the keys' bytes up to about 8 rows, by FMA
// issue beyond: 32 heads on 8, D = 128, 64 single tokens over 1000 to 2000 entries 85 us (4.7 TB/s); 16 and 32 rows, 16
// sequences of up to 4000, 69 and 108 us, as tiles 113 and 187. With 60 and 128 rows tiles are ahead: 6.5 us to
// 11.7 (6 sequences), 326 to 369.
constexpr int WF_KEYS = 16 * (W_THREADS / 32), FEW_W = 32;
constexpr int CARVEOUT_FEW_KB = 40;        // of shared memory, two CTAs' queries: the keys' loads land in the L1 left

__global__ void __launch_bounds__(W_THREADS, 2)
weights_few_kernel(const __grid_constant__ WeightArgs a) {
  constexpr int CH = CACHE_MAX_D / 16;
  __shared__ __align__(16) float sQ[FEW_W][CACHE_MAX_D];
  __shared__ float sL[FEW_W];              // log-sums
  __shared__ int sLim[FEW_W];
  const int tid = threadIdx.x, lane = tid & 31, D = a.D, rows = a.L * a.G;
  const int tiles = (a.S + WF_KEYS - 1) / WF_KEYS, item = blockIdx.x / tiles;
  const int t0 = (blockIdx.x - item * tiles) * WF_KEYS, b = item / a.Hkv, h = item - b * a.Hkv;
  const int len = clamped_len(a, b);
  if (blockIdx.x == 0) {                   // the call's status: the lengths that were clamped
    bool bad = false;
    for (int i = tid; i < a.B; i += W_THREADS) bad |= a.own_len[i] < 0 || a.own_len[i] > a.S;
    bad = __syncthreads_or(bad);
    if (tid == 0) *a.status = bad ? BRISK_ERR_INVALID_ARG : BRISK_OK;
  }
  float sum = 0.f;                         // of key + 8 (lane & 1), over every other row
  const int key = t0 + (tid >> 5) * 16 + (lane >> 2), mine = key + 8 * (lane & 1);
  if (t0 < len) {
    const float* kb = static_cast<const float*>(a.ko.p) + b * a.ko.seq + h * a.ko.head;
    ulonglong2 k[2][CH];
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const int c = 4 * (4 * j + (lane & 3));
        k[e][j] = make_ulonglong2(0, 0);
        if (key + 8 * e < len && c < D) k[e][j] = *reinterpret_cast<const ulonglong2*>(kb + (key + 8 * e) * a.ko.tok + c);
      }
    const int nq = 4 * ((D + 15) / 16);    // pieces of a row (lanes without a piece of a key multiply by zeros)
    const int n = (rows + 1) & ~1;         // an even number of rows, and what they see
    for (int e = tid; e < n * nq; e += W_THREADS) {
      const int r = e / nq, c = 4 * (e - r * nq), row = min(r, rows - 1), i = a.by_G.of(row);
      const float* q = static_cast<const float*>(a.q.p) + b * a.q.seq + i * a.q.tok + (h * a.G + (row - i * a.G)) * a.q.head;
      copy16(&sQ[r][c], c < D ? q + c : q, c < D);
    }
    if (tid < n) {
      int lim = 0;
      float ls = 0.f;
      if (tid < rows) {
        const int i = a.by_G.of(tid);
        const long long token = (long long)b * a.L + i;
        ls = a.lse[token * (a.Hkv * a.G) + h * a.G + (tid - i * a.G)];
        // (a row that saw nothing gives nothing)
        lim = ls == -INFINITY ? 0 : (a.visible ? min(len, a.visible[token]) : len);
      }
      sL[tid] = ls;
      sLim[tid] = lim;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    for (int r = 0; r < rows; r += 2) {
      f32x2 x[2][2];                       // [row][key]: sums over the even and the odd columns
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i >> 1][i & 1] = pack2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        if (16 * j >= D) break;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(&sQ[r + i][4 * (4 * j + (lane & 3))]);
#pragma unroll
          for (int e = 0; e < 2; ++e) x[i][e] = fma2(q.y, k[e][j].y, fma2(q.x, k[e][j].x, x[i][e]));
        }
      }
      float y[2][2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpack2(x[i >> 1][i & 1], lo, hi);
        y[i >> 1][i & 1] = lo + hi;
      }
      // row r + (lane >> 1 & 1), key + 8 (lane & 1)
      const bool up = lane & 2, odd = lane & 1;
      const float z0 = (up ? y[1][0] : y[0][0]) + __shfl_xor_sync(FULL_MASK, up ? y[0][0] : y[1][0], 2);
      const float z1 = (up ? y[1][1] : y[0][1]) + __shfl_xor_sync(FULL_MASK, up ? y[0][1] : y[1][1], 2);
      const float z = (odd ? z1 : z0) + __shfl_xor_sync(FULL_MASK, odd ? z0 : z1, 1);
      const int row = r + (lane >> 1 & 1);
      if (mine < sLim[row]) sum += weight_of(z, a.scale, sL[row]);
    }
  }
  sum += __shfl_xor_sync(FULL_MASK, sum, 2);
  if ((lane & 2) == 0 && mine < a.S) {
    const long long at = (long long)item * a.S + mine;
    if (a.acc_in && mine < len) sum += a.decay * a.acc_in[at];
    a.acc_out[at] = mine < len ? sum : 0.f;
  }
}

// ---------------------------------------------------------------- bf16, on the tensor cores
// S^T = K Q^T: 128 keys are the rows of the product, up to 128 query rows its columns, so that a thread
// holds one key's scores and adds up its weights. The CTAs share the units (sequence, head, key tile)
// evenly. One warp streams key tiles by TMA, one issues the products into four score buffers in TMEM,
// two put blocks of 128 queries with their log-sums into a ring, and two groups of four warps take
// the key tiles in turn. A pass is up to two blocks of queries, which stay, over a run of key tiles: all of a
// fragment where there are no more blocks; else the blocks take turns on runs of CHUNK tiles, and later passes add
// to the sums that the first one wrote. Bound by the keys' bytes up to 128 rows a head; beyond, by the summing warps'
// waits for columns of TMEM (512 rows: tensor cores 36 % active, exponentials 32 %, DRAM 32 %): 64 sequences of 4096
// entries, 8 key heads of 128, 32, 128, 256, 384 and 512 rows a head 93 us (5.8 TB/s), 99, 168, 243 and 324 us (848
// TFLOP/s; when it took 324 without the step below, runs of 8 and 16 tiles 382 and 345, all blocks for every tile 964).
//
// The tensor cores cut a partial sum towards zero at every step of 16 columns: 2.6e-5 of a weight where a score is 128
// positive products of 1, 9e-7 at scores of a few. So with more than 64 columns one step more, after the fourth, adds
// -lse / scale rounded to bf16 (an extra column of the queries, where the keys have 1), and the remainder of the
// log-sum is subtracted afterwards. Partial sums of the scores whose weights count are then above zero first
// and below it later, what is cut off cancels, and what is rounded afterwards is small. 128 rows a head of 72, 80, 96, 112,
// 120 and 128 columns, error against 64 bits in 1e-7: 3.3, 3.8, 1.1, 2.7, 2.3, 2.6; without 7.9, 7.6, 3.0, 13.5, 14.7, 9.0; with
// 64 columns, 3.2 without. It costs 2 to 4 % of the time (128 rows 96.6 -> 98.7 us, 512 rows 318 -> 324; after
// half of the steps in use, whatever their number, some 5 us more).
constexpr int KT = 128, QB = 128, Q_STAGES = 3, CHUNK = 32;
constexpr int WT_THREADS = 384;
constexpr int PANEL = TILE_PANEL;

template <int DP>
struct WShape {
  static constexpr int TILE = KT * DP * 2;
  static constexpr int STAGES = DP == 128 ? 3 : 6;
  static constexpr bool HALF_WAY = DP == 128;      // log-sums come off half-way
  static constexpr int SMEM = 1024 + (Q_STAGES + STAGES) * TILE + (HALF_WAY ? TILE_PANEL : 0);
};

// A pass: nq blocks of queries from q0 on over key tiles [k0, k0 + n); n = 0 after the last.
struct Pass {
  int b, h, k0, n, len, low, last;       // low: entries from here on are hidden from some row; last: the
  int q0, nq, odd;                       // sequence's last tile is among these; odd: number of tiles before, modulo 2
};

// A CTA's passes in order.
struct Passes {
  Walk walk;
  Frag f;
  int at, n, q0, before;                 // tiles of the fragment before this run; the run's; the next block; tiles before the run

  __device__ Passes(const WeightArgs& a, const Plan& plan, const Start& start, int nb) : walk(a, plan, blockIdx.x, start) {
    f.n = at = n = before = 0;
    q0 = nb;
  }
  __device__ bool next(const WeightArgs& a, const Plan& plan, int nb, Pass& p) {
    if (q0 >= nb) {
      at += n;
      before += n;
      q0 = 0;
      if (at >= f.n) {
        if (!walk.next(a, plan, f)) return false;
        at = 0;
      }
      n = nb > 2 ? min(CHUNK, f.n - at) : f.n;
    }
    p = Pass{f.b, f.h, f.k0 + at, n, f.len, 0, f.k0 + at + n == tiles_of(a, f.len), q0, min(2, nb - q0), before & 1};
    q0 += 2;
    return true;
  }
};

template <int DP>
__global__ void __launch_bounds__(WT_THREADS, 1)
weights_tc_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ WeightArgs a) {
  using Sh = WShape<DP>;
  constexpr int STAGES = Sh::STAGES, TILE = Sh::TILE;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = base;
  uint8_t* ring = base + Q_STAGES * TILE;
  uint8_t* extra = ring + STAGES * TILE;           // a panel: 16 more columns of each place of queries, and of any keys
  __shared__ __align__(16) float neg_lse[Q_STAGES][QB];    // -lse but for what the products add, log2 units
  __shared__ __align__(16) int row_lim[Q_STAGES][QB];
  __shared__ uint64_t k_full[STAGES], k_empty[STAGES], q_full[Q_STAGES], q_empty[Q_STAGES];
  __shared__ uint64_t s_full[4], s_empty[4], f_full[2], f_empty[2], done;
  __shared__ Pass info[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int aborted, bad, warp_sum[WT_THREADS / 32];
  __shared__ Start start;
  volatile int* abort_flag = &aborted;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&k_empty[s], 1);
    }
    for (int s = 0; s < Q_STAGES; ++s) {
      mbar_init(&q_full[s], 2);                    // the planning warps
      mbar_init(&q_empty[s], 9);                   // the eight summing warps and the products
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(&s_full[s], 1);
      mbar_init(&s_empty[s], 4);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&f_full[s], 2);
      mbar_init(&f_empty[s], 9);                   // the summing warps and the issuing one
    }
    mbar_init(&done, 1);
    aborted = 0;
    bad = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 0) tmem_alloc(&tmem_slot, 512);
  if constexpr (Sh::HALF_WAY) {
    for (int e = tid; e < TILE_PANEL / 16; e += WT_THREADS) {
      const int r = e >> 3, c = (e ^ r) & 7;       // (a row's 16-byte pieces are swizzled; two a place)
      *reinterpret_cast<uint4*>(extra + e * 16) = make_uint4(c == 2 * Q_STAGES ? 0x3f80u : 0u, 0u, 0u, 0u);
    }
    fence_async_smem();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;

  const int rows = a.L * a.G, nb = (rows + QB - 1) / QB;
  const Plan plan = make_plan<WT_THREADS>(a, blockIdx.x, nullptr, warp_sum, &bad, &start);
  // sequences without entries have no units: zeros everywhere
  for (int b = blockIdx.x; b < a.B; b += gridDim.x)
    if (clamped_len(a, b) == 0)
      for (long long t = tid; t < (long long)a.Hkv * a.S; t += WT_THREADS) a.acc_out[(long long)b * a.Hkv * a.S + t] = 0.f;

  // (a warp that is told that a wait gave up leaves its loop for the barrier at the end)
  auto wait = [&](uint64_t* bar, int phase) { return warp_wait(bar, phase, abort_flag, a.wait_limit); };
  unsigned unit = 0, nf = 0, nq = 0;               // tiles, passes and blocks of queries before
  bool off = false;

  if (warp == 8) {
    Passes passes(a, plan, start, nb);
    Pass f;
    while (!off && passes.next(a, plan, nb, f))
      for (int j = 0; j < f.n; ++j, ++unit) {
        const unsigned st = unit % STAGES;
        off = unit >= STAGES && wait(&k_empty[st], unit / STAGES - 1);
        if (off) break;
        if (elect_one()) {
          mbar_expect_tx(&k_full[st], TILE);
#pragma unroll
          for (int c = 0; c < DP / 64; ++c)
            tma_load_4d(ring + st * TILE + c * PANEL, &map, &k_full[st], c * 64, f.h, (f.k0 + j) * KT, f.b);
        }
        __syncwarp();
      }
    // (whoever reads the tiles may have given up: none is on its way when the CTA ends)
    for (unsigned p = unit > STAGES ? unit - STAGES : 0; p < unit; ++p) mbar_drain(&k_full[p % STAGES], (p / STAGES) & 1);
  } else if (warp == 9) {
    const int nd = (a.D + 15) / 16;
    const uint32_t q_lo = sw128_lo(su32(sQ)), k_lo = sw128_lo(su32(ring)), x_lo = sw128_lo(su32(extra));
    unsigned ns[2] = {0, 0};                       // score buffers a group was given
    auto commit = [&](uint64_t* bar) {
      if (elect_one()) umma_commit(bar);
      __syncwarp();
    };
    while (!off) {
      const unsigned fs = nf & 1;
      off = wait(&f_full[fs], nf >> 1);
      if (off) break;
      const int n = info[fs].n, q0 = info[fs].q0, blocks = info[fs].nq, odd = info[fs].odd;
      __syncwarp();
      if (lane == 0) mbar_arrive(&f_empty[fs]);
      ++nf;
      if (n == 0) break;
      for (int j = 0; j < n && !off; ++j, ++unit) {
        const int g = (odd + j) & 1;
        const unsigned st = unit % STAGES;
        off = wait(&k_full[st], unit / STAGES);
        for (int blk = 0; blk < blocks && !off; ++blk) {
          const unsigned qi = nq + blk, qs = qi % Q_STAGES, buf = 2 * g + (ns[g] & 1);
          off = wait(&q_full[qs], qi / Q_STAGES) || (ns[g] >= 2 && wait(&s_empty[buf], (ns[g] >> 1) - 1));
          if (off) break;
          ++ns[g];
          tc_fence_after();
          const int cols = (min(QB, rows - (q0 + blk) * QB) + 15) & ~15;
          const uint32_t id = idesc_bf16(KT, cols), q = q_lo + qs * (TILE >> 4), k = k_lo + st * (TILE >> 4);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < DP / 16; ++kk) {
              const uint32_t o = (kk >> 2) * (PANEL >> 4) + 2 * (kk & 3);
              if (kk < nd) umma(tmem + buf * 128, sw128(k + o), sw128(q + o), id, kk > 0);
              if (Sh::HALF_WAY && kk == 3) umma(tmem + buf * 128, sw128(x_lo + 2 * Q_STAGES), sw128(x_lo + 2 * qs), id, 1);
            }
            umma_commit(&s_full[buf]);
          }
          __syncwarp();
        }
        if (!off) commit(&k_empty[st]);
      }
      if (off) break;
      for (int blk = 0; blk < blocks; ++blk) commit(&q_empty[(nq + blk) % Q_STAGES]);
      nq += blocks;
    }
    commit(&done);
    mbar_drain(&done, 0);
  } else if (warp >= 10) {
    const int pw = warp - 10;
    Passes passes(a, plan, start, nb);
    for (bool more = true; more && !off;) {
      Pass f{};
      more = passes.next(a, plan, nb, f);
      const unsigned fs = nf & 1;
      const int len = f.len;
      if (nf >= 2 && (off = wait(&f_empty[fs], (nf >> 1) - 1))) break;
      // what no row of the pass is kept from: needed before the first block is there
      int low = len;
      for (int r = f.q0 * QB + lane; r < min(rows, (f.q0 + f.nq) * QB); r += 32) {
        const int i = a.by_G.of(r), g = r - i * a.G;
        const long long token = (long long)f.b * a.L + i;
        if (a.visible) low = min(low, max(0, a.visible[token]));
        if (a.lse[token * (a.Hkv * a.G) + f.h * a.G + g] == -INFINITY) low = 0;
      }
      f.low = __reduce_min_sync(FULL_MASK, low);
      if (pw == 0 && lane == 0) info[fs] = f;
      __syncwarp();
      if (lane == 0) mbar_arrive(&f_full[fs]);
      ++nf;
      for (int x = 0; x < f.nq; ++x, ++nq) {
        const unsigned qs = nq % Q_STAGES;
        const int first = (f.q0 + x) * QB, count = min(QB, rows - first);
        if (nq >= Q_STAGES && (off = wait(&q_empty[qs], nq / Q_STAGES - 1))) break;
        for (int r0 = 32 * pw; r0 < count; r0 += 64) {
          const int r = r0 + lane;
          const __nv_bfloat16* src = nullptr;
          float ls = 0.f;
          int lim = 0;
          if (r < count) {
            const int i = a.by_G.of(first + r), head = f.h * a.G + (first + r - i * a.G);
            const long long token = (long long)f.b * a.L + i;
            src = static_cast<const __nv_bfloat16*>(a.q.p) + f.b * a.q.seq + i * a.q.tok + head * a.q.head;
            ls = a.lse[token * (a.Hkv * a.G) + head];
            lim = a.visible ? min(len, a.visible[token]) : len;
          }
          fetch_queries<DP>(src, a.D, sQ + qs * TILE, r0);
          if (ls == -INFINITY) ls = 0.f, lim = 0;  // a row that saw nothing
          if constexpr (Sh::HALF_WAY) {            // (not where the quotient would be out of bounds, or NaN)
            const float x = -ls / a.scale, added = fabsf(x) < 1e30f ? __bfloat162float(__float2bfloat16_rn(x)) : 0.f;
            *reinterpret_cast<uint32_t*>(extra + r * 128 + ((2 * qs ^ r) & 7) * 16) = __float_as_uint(added) >> 16;
            ls = fmaf(added, a.scale, ls);
          }
          neg_lse[qs][r] = -ls * LOG2E;
          row_lim[qs][r] = lim;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_full[qs]);
      }
    }
  } else {
    const int g = warp >> 2;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const f32x2 scale2 = pack2(a.sl2, a.sl2);
    unsigned ns = 0;
    while (!off) {
      const unsigned fs = nf & 1;
      off = wait(&f_full[fs], nf >> 1);
      if (off) break;
      const Pass x = info[fs];
      __syncwarp();
      if (lane == 0) mbar_arrive(&f_empty[fs]);
      ++nf;
      if (x.n == 0) break;
      float* out = a.acc_out + ((long long)x.b * a.Hkv + x.h) * a.S;
      // later passes add to what the first one left, by the same threads
      const float* in = x.q0 > 0 ? out : (a.acc_in ? a.acc_in + ((long long)x.b * a.Hkv + x.h) * a.S : nullptr);
      const float decay = x.q0 > 0 ? 1.f : a.decay;
      for (int j = 0; j < x.n && !off; ++j) {
        if (((x.odd + j) & 1) != g) continue;
        const int t = (x.k0 + j) * KT + (warp & 3) * 32 + lane, t1 = (x.k0 + j + 1) * KT;
        float old = 0.f;
        if (in && t < x.len) old = in[t];
        f32x2 sum0 = pack2(0.f, 0.f), sum1 = sum0;
        for (int blk = 0; blk < x.nq; ++blk) {
          const unsigned qi = nq + blk, qs = qi % Q_STAGES;
          off = wait(&q_full[qs], qi / Q_STAGES);
          if (off) break;
          const int buf = 2 * g + (ns & 1), count = min(QB, rows - (x.q0 + blk) * QB);
          off = wait(&s_full[buf], ns >> 1);
          if (off) break;
          ++ns;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < count; c += 32) {
            float v[32];
            tmem_ld32(tmem + buf * 128 + lanes + c, v);
            if (x.low < t1 || c + 32 > count) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 ls = *reinterpret_cast<const float4*>(&neg_lse[qs][c + i]);
                const int4 lim = *reinterpret_cast<const int4*>(&row_lim[qs][c + i]);
                const float w0 = ex2(fmaf(v[i], a.sl2, ls.x)), w1 = ex2(fmaf(v[i + 1], a.sl2, ls.y));
                const float w2 = ex2(fmaf(v[i + 2], a.sl2, ls.z)), w3 = ex2(fmaf(v[i + 3], a.sl2, ls.w));
                const int left = count - c - i;
                sum0 = add2(sum0, pack2(t < lim.x && left > 0 ? w0 : 0.f, t < lim.y && left > 1 ? w1 : 0.f));
                sum1 = add2(sum1, pack2(t < lim.z && left > 2 ? w2 : 0.f, t < lim.w && left > 3 ? w3 : 0.f));
              }
            } else {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 ls = *reinterpret_cast<const float4*>(&neg_lse[qs][c + i]);
                float y[4];
                unpack2(fma2(pack2(v[i], v[i + 1]), scale2, pack2(ls.x, ls.y)), y[0], y[1]);
                unpack2(fma2(pack2(v[i + 2], v[i + 3]), scale2, pack2(ls.z, ls.w)), y[2], y[3]);
                sum0 = add2(sum0, pack2(ex2(y[0]), ex2(y[1])));
                sum1 = add2(sum1, pack2(ex2(y[2]), ex2(y[3])));
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&s_empty[buf]);
        }
        if (!off && t < a.S) {
          float y[2];
          unpack2(add2(sum0, sum1), y[0], y[1]);
          out[t] = t < x.len ? fmaf(decay, old, y[0] + y[1]) : 0.f;
        }
      }
      for (int blk = 0; blk < x.nq && !off; ++blk) {
        const unsigned qi = nq + blk, qs = qi % Q_STAGES;
        off = wait(&q_full[qs], qi / Q_STAGES);
        if (!off && lane == 0) mbar_arrive(&q_empty[qs]);
      }
      nq += x.nq;
      if (x.last && x.q0 == 0 && g == 0)           // the places behind the last tile
        for (int t = (x.k0 + x.n) * KT + tid; t < a.S; t += 128) out[t] = 0.f;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
  if (tid == 0 && aborted) set_status(a.status, BRISK_ERR_TIMEOUT);
  if (tid == 0 && blockIdx.x == 0 && bad) set_status(a.status, BRISK_ERR_INVALID_ARG);
}

}  // namespace

cudaError_t launch_weights_tc(const WeightArgs& a, cudaStream_t stream) {
  CUtensorMap map;
  if (!make_cache_map(&map, a.ko, a.D, a.Hkv, a.S, a.B)) return cudaErrorInvalidValue;
  auto run = [&](auto kernel, size_t smem) {
    cudaError_t e = set_up_kernel(kernel, CARVEOUT_FULL_KB, smem);
    if (e != cudaSuccess) return e;
    kernel<<<a.sh.grid_o, WT_THREADS, smem, stream>>>(map, a);
    return cudaGetLastError();
  };
  return a.D > 64 ? run(weights_tc_kernel<128>, WShape<128>::SMEM) : run(weights_tc_kernel<64>, WShape<64>::SMEM);
}

cudaError_t launch_weights_f32(const WeightArgs& a, cudaStream_t stream) {
  auto run = [&](auto kernel, int keys, int carveout, size_t smem) {
    cudaError_t e = set_up_kernel(kernel, carveout, smem);
    if (e != cudaSuccess) return e;
    const long long grid = (long long)a.B * a.Hkv * ((a.S + keys - 1) / keys);
    kernel<<<(unsigned)grid, W_THREADS, smem, stream>>>(a);
    return cudaGetLastError();
  };
  if (a.L * a.G <= FEW_W) return run(weights_few_kernel, WF_KEYS, CARVEOUT_FEW_KB, 0);
  return run(weights_simt_kernel, W_KEYS, CARVEOUT_FULL_KB, sizeof(float) * (W_KEYS * WS + W_ROWS * CACHE_MAX_D + 2 * W_ROWS));
}

}  // namespace brisk
