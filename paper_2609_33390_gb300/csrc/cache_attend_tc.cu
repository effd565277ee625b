// bf16 attention over a shared prefix and own caches on the tensor cores of sm_103a.
//
// One CTA an SM works through its share of the (row tile, key tile) units (see Plan). Two groups of
// four warps hold a slot each: 128 query rows, a row a thread, with its scores S and sum of values
// O in TMEM. One thread streams key and value tiles (128 entries) through a ring by TMA; one
// thread issues S = Q K^T (both operands in shared memory), and, when the slot's threads have put
// P = exp2(S - m) into TMEM as bf16 over S, O += P V (P from TMEM, V from shared memory as it lies, its
// columns contiguous). A tile of more than 128 rows fills both slots and every key tile serves both
// (`pair`); with fewer rows the slots take the key tiles in turn and their sums are joined at the end.
// While one slot's threads take exponentials the tensor cores work for the other.
//
// The maximum a row subtracts is held back until a score exceeds it by 2^8: P and the sums then stay
// below 2^8 times their number, and O is seldom rescaled. Rounding P to bf16 costs at most 2^-9 of each
// weight, as much as rounding the result; sums are fp32.
//
// Entries that a row must not see: scores are masked by selection; a value row that some row of the
// tile does not see gets weight 0 there, which a NaN or an infinity would defeat, so such values are
// set to 0 in shared memory and added at the end to the rows that see them.
//
// Every wait on an mbarrier is bounded; a CTA that gave up goes through the rest of its work without
// waiting or issuing anything, reports BRISK_ERR_TIMEOUT and frees its TMEM after what it had issued.
#include "cache.cuh"
#include "tensor_core.cuh"

namespace brisk {
namespace {

constexpr int KT = ATTEND_KT_TC, RT = ATTEND_RT_TC, SLOT = 128;
constexpr int SOFT_THREADS = 2 * SLOT;
constexpr int ATT_THREADS = SOFT_THREADS + 128;    // and a copying, an issuing two issuing and a planning warp
constexpr float LAZY = 8.f;                        // log2 of what a score may exceed the held maximum by
constexpr uint32_t TMEM_COLS = 512;                // S0 | S1 | O0 | O1, 128 columns each
constexpr int PANEL = KT * 128;                    // bytes of 64 columns of a tile

struct AttendMaps { CUtensorMap kp, vp, ko, vo; };

template <int DP>
struct Shape {
  static constexpr int TILE = KT * DP * 2;         // bytes of a tile of 128 rows
  static constexpr int STAGES = DP == 128 ? 4 : 8;
  static constexpr int SMEM = 1024 + (2 + STAGES) * TILE + (CACHE_MAX_B + 1) * 4;
};

// Places of the key and value tiles of a fragment of n tiles in the ring's order, which is the order
// in which the issuing thread takes them.
__device__ __forceinline__ int k_place(bool pair, int j) { return pair ? 2 * j : (j == 0 ? 0 : 2 * j - 1); }
__device__ __forceinline__ int v_place(bool pair, int j, int n) {
  return pair ? 2 * j + 1 : (j < n - 1 ? 2 * j + 2 : 2 * n - 1);
}

__device__ __forceinline__ bool odd_bf16x2(uint32_t x) {   // an infinity or NaN among the two
  return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t without_odd(uint32_t x) {
  if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
  if ((x & 0x7f800000u) == 0x7f800000u) x &= 0x0000ffffu;
  return x;
}

// Adds the infinities and NaN of the own values t0 <= t < t1 to the columns of a row that its thread has
// stored: to a part's (by groups of four, `per` apart) or to the result's. Out of the way: it is seldom run.
__device__ __noinline__ void add_odd(const AttendArgs& a, int b, int h, int t0, int t1, int c, int c1, float* part,
                                     int per, __nv_bfloat16* out) {
  for (; c < c1; ++c) {
    float sum = 0.f;
    for (int t = t0; t < t1; ++t) {
      const float x = __bfloat162float(*(static_cast<const __nv_bfloat16*>(a.vo.p) + b * a.vo.seq + t * a.vo.tok +
                                         h * a.vo.head + c));
      if (!isfinite(x)) sum += x;
    }
    if (sum == 0.f) continue;
    if (part) part[(long long)(c & ~3) * per + (c & 3)] += sum;
    else out[c] = __float2bfloat16_rn(__bfloat162float(out[c]) + sum);
  }
}

// What the planning warps tell the others of a fragment.
struct FragInfo {
  Frag f;
  int len;                                         // entries of the prefix, or in use of the own cache
  int low;                                         // entries from here on are hidden from some row
};

template <int DP>
__global__ void __launch_bounds__(ATT_THREADS, 1)
attend_tc_kernel(const __grid_constant__ AttendMaps maps, const __grid_constant__ AttendArgs a) {
  using Sh = Shape<DP>;
  constexpr int STAGES = Sh::STAGES, TILE = Sh::TILE, VPR = DP / 8;   // 16-byte pieces of a row
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = base;                              // [2][DP / 64][128 rows][128 B], swizzled
  uint8_t* ring = base + 2 * TILE;
  int32_t* cum = reinterpret_cast<int32_t*>(ring + STAGES * TILE);
  __shared__ uint64_t full[STAGES], empty[STAGES], s_full[2], p_ready[2][2], o_full[2];
  __shared__ uint64_t frag_full[2], frag_empty[2], q_free[2], turn[2], slots, done;
  __shared__ FragInfo info[2];
  __shared__ int row_id[2][RT], row_lim[2][RT];    // token * Hq + head (its complement: padding), keys seen
  __shared__ uint32_t tmem_slot;
  __shared__ int aborted, bad, warp_sum[ATT_THREADS / 32], odd_of[2][8];
  __shared__ float2 ml_of[2][2][SLOT];
  volatile int* abort_flag = &aborted;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 2);                     // both slots' products
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&s_full[s], 1);
      mbar_init(&p_ready[s][0], 4);                // a lane of each of the slot's warps, for either half
      mbar_init(&p_ready[s][1], 4);
      mbar_init(&o_full[s], 1);
      mbar_init(&frag_full[s], 1);
      mbar_init(&frag_empty[s], 8);                // the slots' warps
      mbar_init(&q_free[s], 2);
      mbar_init(&turn[s], 1);
    }
    mbar_init(&slots, 8);
    mbar_init(&done, 2);
    aborted = 0;
    bad = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 0) tmem_alloc(&tmem_slot, TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;

  const int own = count_tiles<ATT_THREADS>(a, KT, cum, warp_sum, &bad);
  const Plan plan(a, RT, KT, own);
  if (blockIdx.x == 0)
    for (int b = tid; b <= a.B; b += ATT_THREADS) a.cum[b] = cum[b];

  // (a warp that is told that a wait gave up leaves its loop for the barrier at the end)
  auto wait = [&](uint64_t* bar, int phase) { return warp_wait(bar, phase, abort_flag, a.wait_limit); };
  int pos = 0;                                     // ring places of the fragments before this one
  int nf = 0;                                      // fragments before this one: it uses the words nf & 1

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 8) {
      // copies: a key or value tile at a time, in the ring's order
      Walk walk(plan, cum, blockIdx.x);
      Frag f;
      int issued = 0;
      bool off = false;
      while (!off && walk.next(plan, cum, f)) {
        const bool pair = f.rows > SLOT;
        const CUtensorMap* mk = f.prefix ? &maps.kp : &maps.ko;
        const CUtensorMap* mv = f.prefix ? &maps.vp : &maps.vo;
        int nk = 0, nv = 0;
        for (int i = 0; i < 2 * f.n; ++i) {
          const bool key = nk < f.n && k_place(pair, nk) == i;
          const int t0 = (f.k0 + (key ? nk++ : nv++)) * KT;
          const unsigned p = pos + i, st = p % STAGES;
          off = p >= STAGES && wait(&empty[st], p / STAGES - 1);
          if (off) break;
          if (elect_one()) {
            mbar_expect_tx(&full[st], TILE);
#pragma unroll
            for (int c = 0; c < DP / 64; ++c)
              tma_load_4d(ring + st * TILE + c * PANEL, key ? mk : mv, &full[st], c * 64, f.h, t0, f.b);
          }
          __syncwarp();
          issued = (int)p + 1;
        }
        pos += 2 * f.n;
      }
      if (off)
        for (int p = issued > STAGES ? issued - STAGES : 0; p < issued; ++p)
          mbar_drain(&full[p % STAGES], (p / STAGES) & 1);
    } else if (warp != 10) {
      // products of a slot, issued by one lane; the warp stays together around it. A warp a slot: one's
      // waits do not keep the tensor cores from the other's products. Both go through every place of the
      // ring in order, also through those that only the other one reads, and both hand it back: a barrier's
      // phase is known by its parity alone, so that none may be left out.
      const int s = warp == 9 ? 0 : 1;
      const int nd = (a.D + 15) / 16;              // 16 columns a step of Q K^T, and a unit of O's width
      const uint32_t id_s = idesc_bf16(SLOT, KT), id_o = idesc_bf16(SLOT, 16 * nd) | IDESC_B_MN;
      const uint32_t q_lo = sw128_lo(su32(sQ)), k_lo = sw128_lo(su32(ring)), v_lo = sw128_lo_mn(su32(ring), PANEL);
      const uint32_t tS = tmem + s * 128, tO = tmem + 256 + s * 128;
      unsigned cur = 0;                            // ring places taken
      int nready = 0, nturn = 0;
      const unsigned places = 2 * plan.units_of(blockIdx.x);
      bool off = false;                            // a wait gave up: nothing more is issued
      for (; cur < places && !off; ++nf) {
        const int fs = nf & 1;
        off = wait(&frag_full[fs], nf >> 1);
        if (off) break;
        tc_fence_after();
        const int n = info[fs].f.n, k0 = info[fs].f.k0, len = info[fs].len;
        const bool pair = info[fs].f.rows > SLOT;
        const int step = pair ? 1 : 2;
        const uint32_t q = q_lo + (pair ? s : fs) * (TILE >> 4);
        int left = pair ? n : (n + 1 - s) / 2;     // tiles of the slot whose scores are still to come
        if (left == 0 && elect_one()) umma_commit(&q_free[fs]);
        __syncwarp();
        bool begun = false;
        for (int j = -step; j < n; ++j) {          // values of tile j, scores of tile j + step
          const bool any = j >= 0, more = j + step < n;
          unsigned sv = 0, sk = 0;
          if (any) {
            sv = cur % STAGES;
            off = wait(&full[sv], cur / STAGES);
            ++cur;
          }
          if (more && !off) {
            sk = cur % STAGES;
            off = wait(&full[sk], cur / STAGES);
            ++cur;
          }
          if (off) break;
          if (!pair && (j & 1) != s) {
            if (lane == 0) {
              if (any) mbar_arrive(&empty[sv]);
              if (more) mbar_arrive(&empty[sk]);
            }
            __syncwarp();
            continue;
          }
          const uint32_t v = v_lo + sv * (TILE >> 4), k = k_lo + sk * (TILE >> 4);
          const int steps = (len - (k0 + j) * KT + 15) / 16;   // of 16 keys: entries in use
          if (any) {
            off = wait(&p_ready[s][0], nready);
            // a pair's products go slot by slot: taken together, both slots would get their scores, and
            // take their exponentials, at the same time, and then wait at the same time
            if (pair && !off && (s == 1 || nturn > 0)) off = wait(&turn[s], nturn - 1 + s);
            if (off) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int kk = 0; kk < KT / 32; ++kk)
                if (kk < steps) umma_ts(tO, tS + 8 * kk, sw128(v + kk * 128), id_o, begun || kk > 0);
            }
            __syncwarp();
            off = wait(&p_ready[s][1], nready++);
            if (off) break;
            begun = true;
          }
          tc_fence_after();
          --left;
          if (elect_one()) {
            if (any) {
#pragma unroll
              for (int kk = KT / 32; kk < KT / 16; ++kk)
                if (kk < steps) umma_ts(tO, tS + 8 * kk, sw128(v + kk * 128), id_o, 1);
              umma_commit(&empty[sv]);
              if (!more) umma_commit(&o_full[s]);
            }
            if (more) {
#pragma unroll
              for (int kk = 0; kk < DP / 16; ++kk) {
                const uint32_t o = (kk >> 2) * (PANEL >> 4) + 2 * (kk & 3);
                if (kk < nd) umma(tS, sw128(q + o), sw128(k + o), id_s, kk > 0);
              }
              umma_commit(&s_full[s]);
              umma_commit(&empty[sk]);
              if (left == 0) umma_commit(&q_free[fs]);
            }
            if (pair && any) mbar_arrive(&turn[s ^ 1]);
          }
          __syncwarp();
          if (any) ++nturn;
        }
      }
      if (elect_one()) umma_commit(&done);
      mbar_drain(&done, 0);
    } else {
      // plan: the fragments in turn, their rows and their queries, one fragment ahead of the products
      const int np = 2 * ((a.D + 15) / 16);        // 16-byte pieces that the products read
      Walk walk(plan, cum, blockIdx.x);
      FragInfo x;
      bool was_pair = false;
      while (walk.next(plan, cum, x.f)) {
        const int fs = nf & 1;
        const bool pair = x.f.rows > SLOT;
        x.len = x.f.prefix ? a.P : clamped_len(a, x.f.b);
        if (nf >= 2 && (wait(&frag_empty[fs], (nf >> 1) - 1) || wait(&q_free[fs], (nf >> 1) - 1))) break;
        if (nf >= 1 && (pair || was_pair) && wait(&q_free[fs ^ 1], (nf - 1) >> 1)) break;
        was_pair = pair;
        x.low = x.len;
        for (int r0 = 0; r0 < x.f.rows; r0 += 32) {
          const int r = r0 + lane;
          const __nv_bfloat16* src = nullptr;
          int token = 0, id = 0;
          if (r < x.f.rows) {
            int head;
            row_of(a, x.f, r, token, head);
            const int b = token / a.L, i = token - b * a.L;
            id = token * (a.Hkv * a.G) + head;
            src = static_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.seq + i * a.q.tok + head * a.q.head;
          }
          // 4 lanes a row, 64 bytes of it at a time: the queries of 32 rows, eight at a time
          const int last = min(32, x.f.rows - r0), q4 = lane & 3;
#pragma unroll 1
          for (int i = 0; i < last; i += 8) {
            const int in = i + (lane >> 2), at = (r0 & (SLOT - 1)) + in;
            const unsigned long long from = __shfl_sync(FULL_MASK, reinterpret_cast<unsigned long long>(src), in);
            const uint32_t to = su32(sQ + (pair ? r0 >> 7 : fs) * TILE + at * 128);
            if (in < last)
#pragma unroll
              for (int k = 0; k < VPR / 4; ++k) {
                const int c = 4 * k + q4;
                const uint32_t dst = to + (c >> 3) * PANEL + ((c ^ at) & 7) * 16;
                if (8 * c < a.D)
                  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(from + 16 * c) : "memory");
                else if (c < np)
                  asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(dst), "r"(0) : "memory");
              }
          }
          if (r < x.f.rows) {
            const int lim = row_limit(a, x.f, token, x.len);
            const bool idle = row_idle(a, token);
            row_id[fs][r] = idle ? ~id : id;
            row_lim[fs][r] = lim;
            if (!idle) x.low = min(x.low, lim);
          }
        }
        x.low = __reduce_min_sync(FULL_MASK, x.low);
        if (lane == 0) info[fs] = x;
        asm volatile("cp.async.wait_all;" ::: "memory");
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&frag_full[fs]);
        ++nf;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int s = warp >> 2, r = tid & (SLOT - 1), D = a.D;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + s * 128 + lanes, tO = tmem + 256 + lanes;
    const int places = 2 * plan.units_of(blockIdx.x);
    int nS = 0, nO = 0, nsync = 0;                 // tiles and fragments this slot had; meetings of the slots
    bool off = false;
    auto meet = [&]() {                            // both slots' warps
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&slots);
      off = wait(&slots, nsync++);
      tc_fence_after();
    };
    for (; pos < places && !off; ++nf) {
      const int fs = nf & 1;
      off = wait(&frag_full[fs], nf >> 1);
      if (off) break;
      const Frag& f = info[fs].f;
      const int len = info[fs].len, low = info[fs].low, n = f.n, k0 = f.k0;
      const bool pair = f.rows > SLOT;
      const int my = pair ? s * SLOT + r : r;      // this thread's row
      const bool mine = my < f.rows;
      const int lim = mine ? row_lim[fs][my] : 0;
      const bool warp_live = __any_sync(FULL_MASK, mine);
      if (lane == 0) odd_of[fs][warp] = 0;

      float m = -INFINITY, l = 0.f;
      int tiles = 0;
      for (int j = pair ? 0 : s; j < n; j += pair ? 1 : 2, ++tiles) {
        const int t0 = (k0 + j) * KT, end = min(len - t0, KT);     // entries in use of the tile
        off = wait(&s_full[s], nS++);
        if (off) break;
        tc_fence_after();
        // values that some row does not see, and those behind the last entry that the last step reads
        const int v0 = max(low - t0, 0), v1 = min((end + 15) & ~15, KT);
        if (v0 < v1) {
          const int pl = pos + v_place(pair, j, n), st = pl % STAGES;
          off = wait(&full[st], pl / STAGES);
          if (off) break;
          bool odd = false;
#pragma unroll 1
          for (int e = r; e < (v1 - v0) * VPR; e += SLOT) {
            const int row = v0 + e / VPR, c = e % VPR;
            uint4* at = reinterpret_cast<uint4*>(ring + st * TILE + (c >> 3) * PANEL + row * 128 +
                                                 ((c & 7) ^ (row & 7)) * 16);
            const uint4 x = *at;
            if (odd_bf16x2(x.x) || odd_bf16x2(x.y) || odd_bf16x2(x.z) || odd_bf16x2(x.w)) {
              *at = make_uint4(without_odd(x.x), without_odd(x.y), without_odd(x.z), without_odd(x.w));
              odd |= row < end;
            }
          }
          if (__any_sync(FULL_MASK, odd) && lane == 0) odd_of[fs][warp] = 1;
          fence_async_smem();                      // (the product waits for all four warps)
        }
        auto ready = [&](int half) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_ready[s][half]);
        };
        if (warp_live) {
          float v[KT];
          tmem_ld128(tS, v);
          if (__any_sync(FULL_MASK, mine && lim - t0 < KT)) {
            const int seen_here = lim - t0;
#pragma unroll
            for (int c = 0; c < KT; ++c) v[c] = c < seen_here ? v[c] : -INFINITY;
          }
          float top[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int c = 4; c + 8 <= KT; c += 8)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[i] = fmaxf(fmaxf(top[i], v[c + i]), v[c + 4 + i]);
#pragma unroll
          for (int i = 0; i < 4; ++i) top[i] = fmaxf(top[i], v[KT - 4 + i]);
          const float t = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.sl2;
          if (__any_sync(FULL_MASK, t > m + LAZY)) {
            const float mn = fmaxf(m, t), alpha = ex2(m - (mn == -INFINITY ? 0.f : mn));
            m = mn;
            l *= alpha;
            if (tiles > 0)
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                float o[16];
                tmem_ld16(tO + s * 128 + c, o);
                uint32_t x[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(o[i] * alpha);
                tmem_st16(tO + s * 128 + c, x);
              }
          }
          const float ms = m == -INFINITY ? 0.f : m;
          const f32x2 scale2 = pack2(a.sl2, a.sl2), minus2 = pack2(-ms, -ms);
          f32x2 sum0 = pack2(0.f, 0.f), sum1 = sum0;
#pragma unroll
          for (int c0 = 0; c0 < KT; c0 += 32) {
            uint32_t p[16];
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
              float x[4];
              unpack2(fma2(pack2(v[c0 + c], v[c0 + c + 1]), scale2, minus2), x[0], x[1]);
              unpack2(fma2(pack2(v[c0 + c + 2], v[c0 + c + 3]), scale2, minus2), x[2], x[3]);
#pragma unroll
              for (int i = 0; i < 4; ++i) x[i] = ex2(x[i]);
              sum0 = add2(sum0, pack2(x[0], x[1]));
              sum1 = add2(sum1, pack2(x[2], x[3]));
              const __nv_bfloat162 h0 = __floats2bfloat162_rn(x[0], x[1]), h1 = __floats2bfloat162_rn(x[2], x[3]);
              p[c / 2] = *reinterpret_cast<const uint32_t*>(&h0);
              p[c / 2 + 1] = *reinterpret_cast<const uint32_t*>(&h1);
            }
            tmem_st16(tS + c0 / 2, p);
            if (c0 == 32) {                        // half of the keys: their product may begin
              tmem_st_wait();
              ready(0);
            }
          }
          float x[2];
          unpack2(add2(sum0, sum1), x[0], x[1]);
          l += x[0] + x[1];
          tmem_st_wait();
        } else {
          ready(0);
        }
        ready(1);
      }
      if (off || (tiles > 0 && (off = wait(&o_full[s], nO++)))) break;
      tc_fence_after();
      float w0 = 1.f, w1 = 0.f;                    // weights of this slot's sums, and of the other's
      if (!pair) ml_of[fs][s][r] = make_float2(m, l);
      // for the other slot's sums, or to know what its warps found among the values
      const bool cleaned = !f.prefix && low < len;
      if (!pair || cleaned) meet();
      if (off) break;
      if (!pair) {
        const float2 x = ml_of[fs][0][r], y = ml_of[fs][1][r];
        m = fmaxf(x.x, y.x);
        const float ms = m == -INFINITY ? 0.f : m;
        w0 = x.x == m ? 1.f : ex2(x.x - ms);
        w1 = y.x == m ? 1.f : ex2(y.x - ms);
        l = w0 * x.y + w1 * y.y;
      }
      int odd = 0;
      if (cleaned)
        for (int w = 0; w < 8; ++w) odd |= odd_of[fs][w];

      if (warp_live) {
        const int id = mine ? row_id[fs][my] : -1, row = id < 0 ? ~id : id;
        const bool whole = f.whole, none = l == 0.f || id < 0;
        const float inv = none ? 0.f : 1.f / l;
        const int per = min(RT, f.prefix ? plan.R : plan.LG);
        float* part = (f.prefix ? a.part_p : a.part_o) + part_at(f.slot, per, D, my, 0);
#pragma unroll 1
        for (int c = pair ? 0 : 16 * s; c < D; c += pair ? 16 : 32) {
          float o[16];
          tmem_ld16(tO + (pair ? s * 128 : 0) + c, o);
          if (!pair && n > 1) {
            float y[16];
            tmem_ld16(tO + 128 + c, y);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = fmaf(w1, y[i], w0 * o[i]);
          }
          if (mine) {
            if (whole) {
              __nv_bfloat16* to = static_cast<__nv_bfloat16*>(a.out) + (long long)row * D + c;
#pragma unroll
              for (int i = 0; i < 16; i += 8)
                if (c + i < D) {
                  uint32_t x[4];
#pragma unroll
                  for (int k = 0; k < 4; ++k) {
                    const __nv_bfloat162 h = none ? __floats2bfloat162_rn(0.f, 0.f)
                                                  : __floats2bfloat162_rn(o[i + 2 * k] * inv, o[i + 2 * k + 1] * inv);
                    x[k] = *reinterpret_cast<const uint32_t*>(&h);
                  }
                  *reinterpret_cast<uint4*>(to + i) = make_uint4(x[0], x[1], x[2], x[3]);
                }
            } else {
#pragma unroll
              for (int i = 0; i < 16; i += 4)
                if (c + i < D) store4(part + (long long)(c + i) * per, make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]));
            }
            if (odd && !none)
              add_odd(a, f.b, f.h, max(low, k0 * KT), min(lim, (k0 + n) * KT), c, min(c + 16, D), whole ? nullptr : part,
                      per, static_cast<__nv_bfloat16*>(a.out) + (long long)row * D);
          }
          __syncwarp();
        }
        if (mine && (pair || s == 0)) {
          if (!whole) (f.prefix ? a.ml_p : a.ml_o)[(long long)f.slot * per + my] = make_float2(m, l);
          else if (a.lse) a.lse[row] = none ? -INFINITY : (m + log2f(l)) * (1.f / LOG2E);
        }
      }
      if (!pair) meet();                           // both slots have read both sums
      __syncwarp();
      if (lane == 0) mbar_arrive(&frag_empty[fs]);
      pos += 2 * n;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, TMEM_COLS);
  if (tid == 0)
    a.errs[blockIdx.x] = aborted ? BRISK_ERR_TIMEOUT : (bad && blockIdx.x == 0 ? BRISK_ERR_INVALID_ARG : BRISK_OK);
}

}  // namespace

// Tiles of 64 columns x 128 entries of one head and sequence, 128-byte swizzle, zeros outside.
bool make_cache_map(CUtensorMap* map, const CacheView& v, int D, int heads, int toks, int seqs) {
  if (!v.p) {                                      // no such entries: never read
    *map = CUtensorMap{};
    return true;
  }
  auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[4] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(heads),
                        static_cast<cuuint64_t>(toks), static_cast<cuuint64_t>(seqs)};
  cuuint64_t strides[3] = {static_cast<cuuint64_t>(v.head) * 2, static_cast<cuuint64_t>(v.tok) * 2,
                           static_cast<cuuint64_t>(v.seq) * 2};
  cuuint32_t box[4] = {64, 1, KT, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(v.p), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t stream) {
  AttendMaps maps;
  if (!make_cache_map(&maps.kp, a.kp, a.D, a.Hkv, a.P, 1) || !make_cache_map(&maps.vp, a.vp, a.D, a.Hkv, a.P, 1) ||
      !make_cache_map(&maps.ko, a.ko, a.D, a.Hkv, a.S, a.B) || !make_cache_map(&maps.vo, a.vo, a.D, a.Hkv, a.S, a.B))
    return cudaErrorInvalidValue;
  auto run = [&](auto kernel, size_t smem) {
    cudaError_t e = set_up_kernel(kernel, CARVEOUT_FULL_KB, smem);
    if (e != cudaSuccess) return e;
    kernel<<<a.grid, ATT_THREADS, smem, stream>>>(maps, a);
    return cudaGetLastError();
  };
  return a.D > 64 ? run(attend_tc_kernel<128>, Shape<128>::SMEM) : run(attend_tc_kernel<64>, Shape<64>::SMEM);
}

}  // namespace brisk
