// bf16 attention over a shared prefix and own caches on the tensor cores of sm_103a.
//
// A slot is 128 query rows of a key head: four warps, a row a thread, and scores S and a sum of values O of
// 128 columns each in TMEM. One thread streams key and value tiles (128 entries) through a ring by TMA; one
// thread issues S = Q K^T (both operands in shared memory), and, when the slot's threads have put
// P = exp2(S - m) into TMEM as bf16 over S, O += P V (P from TMEM, V from shared memory as it lies, its
// columns contiguous). A slot's products and exponentials take turns, so two slots share an SM: one's
// threads take exponentials while the tensor cores work for the other.
//
// attend_pair_kernel, over the prefix: one CTA an SM with two slots, 256 rows, that share every tile. Bound
// by the tensor cores (active 70 % of the time) and the exponentials' way between them: 128 blocks of 32 positions, 32
// heads on 8, D = 128, over 8192 entries 320 us, 1.7 PFLOP/s.
// attend_slot_kernel, over the own caches (and over the prefix where it has few units, see divide): two
// CTAs an SM, each working through fragments of its own. Bound by the entries' bytes where the caches are
// long (256 single tokens over 512 to 2048 entries each, 222 us, 6 TB/s), by what a fragment costs around its
// tiles where they are short (a block of 32 positions over 4096 and 1100 entries: 14 us for two tiles a CTA; 128 blocks
// over 256 to 1024 own entries each: 97 us, where their bytes and the parts' take 62).
// The CTAs share the units of work evenly (see Plan). Where both kernels run, the own caches' is first; the
// prefix's takes over SM by SM and joins the own entries' parts at the end of its fragments, which are long.
//
// The maximum a row subtracts is held back until a score exceeds it by 2^8: P and the sums then stay
// below 2^8 times their number, and O is seldom rescaled (128 blocks as above, own entries too: 437 us, 479 with the
// exact maximum). Rounding P to bf16 costs at most 2^-8 of each
// weight, as much as rounding the result; sums are fp32.
//
// Entries that a row must not see: scores are masked by selection; a value row that some row of the
// tile does not see gets weight 0 there, which a NaN or an infinity would defeat, so such values are
// set to 0 in shared memory and added at the end to the rows that see them.
//
// Every wait on an mbarrier is bounded; a warp that is told that a wait of the CTA gave up leaves its loop
// for the barrier at the end, and the CTA reports BRISK_ERR_TIMEOUT and frees its TMEM after what it had
// issued. A barrier's phase is known by its parity alone: whoever waits on one waits for all its phases.
#include "attend_tc.cuh"

namespace brisk {
namespace {

using Weight = WeightAs<__nv_bfloat16>;

struct AttendMaps { CUtensorMap k, v, k2, v2; };   // of a kernel's first and second caches

__device__ __forceinline__ bool odd_bf16x2(uint32_t x) {   // an infinity or NaN among the two
  return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t without_odd(uint32_t x) {
  if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
  if ((x & 0x7f800000u) == 0x7f800000u) x &= 0x0000ffffu;
  return x;
}

// Sets to 0 the infinities and NaN among the values of rows v0 <= row < v1 of a tile, by a slot's 128
// threads; true where one of them lies before `end`.
template <int DP>
__device__ __forceinline__ bool clean_values(uint8_t* tile, int v0, int v1, int end, int tid) {
  constexpr int VPR = DP / 8;                      // 16-byte pieces of a row
  bool odd = false;
#pragma unroll 2
  for (int e = tid; e < (v1 - v0) * VPR; e += SLOT) {
    const int row = v0 + e / VPR, c = e % VPR;
    uint4* at = reinterpret_cast<uint4*>(tile + (c >> 3) * PANEL + row * 128 + ((c & 7) ^ (row & 7)) * 16);
    const uint4 x = *at;
    if (odd_bf16x2(x.x) || odd_bf16x2(x.y) || odd_bf16x2(x.z) || odd_bf16x2(x.w)) {
      *at = make_uint4(without_odd(x.x), without_odd(x.y), without_odd(x.z), without_odd(x.w));
      odd |= row < end;
    }
  }
  fence_async_smem();
  return odd;
}

// Adds the infinities and NaN of the own values t0 <= t < t1 to the columns of a row that its thread has
// stored: to a part's (by groups of four, `per` apart) or to the result's. Out of the way: it is seldom run.
__device__ __noinline__ void add_odd(const AttendArgs& a, int b, int h, int t0, int t1, float* part, int per,
                                     __nv_bfloat16* out) {
  for (int c = 0; c < a.D; ++c) {
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

template <int DP>
__device__ __forceinline__ void load_tile(uint8_t* to, const CUtensorMap* map, uint64_t* bar, int h, int t0, int b) {
  mbar_expect_tx(bar, KT * DP * 2);
#pragma unroll
  for (int c = 0; c < DP / 64; ++c) tma_load_4d(to + c * PANEL, map, bar, c * 64, h, t0, b);
}

// ---------------------------------------------------------------- two slots a CTA, over the prefix
constexpr int PAIR_THREADS = 2 * SLOT + 128;       // and a copying and two issuing warps (and one idle)
template <int DP>
struct PairShape {
  static constexpr int TILE = KT * DP * 2;         // bytes of a tile of 128 rows
  static constexpr int STAGES = DP == 128 ? 4 : 8;
  static constexpr int SMEM = 1024 + (2 + STAGES) * TILE + 8 * STAGE_BYTES;
};

template <int DP>
__global__ void __launch_bounds__(PAIR_THREADS, 1)
attend_pair_kernel(const __grid_constant__ AttendMaps maps, const __grid_constant__ AttendArgs a) {
  constexpr int STAGES = PairShape<DP>::STAGES, TILE = PairShape<DP>::TILE;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* sQ = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t *ring = sQ + 2 * TILE, *stage = ring + STAGES * TILE;
  __shared__ uint64_t full[STAGES], empty[STAGES], s_full[2], p_ready[2][2], o_full[2], q_full[2], turn[2], done;
  __shared__ uint32_t tmem_slot;
  __shared__ int aborted;
  volatile int* abort_flag = &aborted;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 2);                     // both slots' products
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&s_full[s], 1);
      mbar_init(&p_ready[s][0], 4);                // the slot's warps, for either half of the keys
      mbar_init(&p_ready[s][1], 4);
      mbar_init(&o_full[s], 1);
      mbar_init(&q_full[s], 4);
      mbar_init(&turn[s], 1);
    }
    mbar_init(&done, 2);
    aborted = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 0) tmem_alloc(&tmem_slot, 512);      // S0 | S1 | O0 | O1
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  let_next_begin();
  const uint32_t tmem = tmem_slot;
  auto wait = [&](uint64_t* bar, int phase) { return warp_wait(bar, phase, abort_flag, a.wait_limit); };

  const int R = a.B * a.L * a.G, kP = (a.P + KT - 1) / KT, nPT = (R + PAIR_ROWS - 1) / PAIR_ROWS;
  const int UP = a.Hkv * nPT * kP, share = (UP + a.sh.grid_p - 1) / a.sh.grid_p;
  const int2 range = units_of(blockIdx.x, share, UP);
  int u = range.x;
  bool off = false;                                // a wait gave up

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    unsigned cur = 0;                              // ring places taken: key and value tiles in turn
    if (warp == 8) {
      for (; u < range.y && !off; ++u) {
        const int item = u / kP, t0 = (u - item * kP) * KT, h = item / nPT;
#pragma unroll 1
        for (int i = 0; i < 2; ++i, ++cur) {
          const unsigned st = cur % STAGES;
          off = cur >= STAGES && wait(&empty[st], cur / STAGES - 1);
          if (off) break;
          if (elect_one()) load_tile<DP>(ring + st * TILE, i ? &maps.v : &maps.k, &full[st], h, t0, 0);
          __syncwarp();
        }
      }
      // (whoever reads the tiles may have given up: none is on its way when the CTA ends)
      for (unsigned p = cur > STAGES ? cur - STAGES : 0; p < cur; ++p) mbar_drain(&full[p % STAGES], (p / STAGES) & 1);
    } else if (warp < 11) {
      // products of a slot, issued by one lane; the warp stays together around it. A warp a slot: one's
      // waits do not keep the tensor cores from the other's products.
      const int s = warp - 9, nd = (a.D + 15) / 16;   // 16 columns a step of Q K^T, and a unit of O's width
      const uint32_t id_o = idesc_bf16(SLOT, 16 * nd) | IDESC_B_MN;
      const uint32_t q = sw128_lo(su32(sQ + s * TILE)), k_lo = sw128_lo(su32(ring)), v_lo = sw128_lo_mn(su32(ring), PANEL);
      const uint32_t tS = tmem + s * 128, tO = tmem + 256 + s * 128;
      int nready = 0, nf = 0;
      while (u < range.y && !off) {
        const int n = min(kP - u % kP, range.y - u), k0 = u % kP;
        off = wait(&q_full[s], nf++);
        for (int j = -1; j < n && !off; ++j) {     // values of tile j, scores of tile j + 1
          const bool any = j >= 0, more = j + 1 < n;
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
          const uint32_t v = v_lo + sv * (TILE >> 4), k = k_lo + sk * (TILE >> 4);
          const int steps = (a.P - (k0 + j) * KT + 15) / 16;
          if (any) {
            off = wait(&p_ready[s][0], nready);
            // the products go slot by slot: taken together, both slots would get their scores, and take
            // their exponentials, at the same time, and then wait at the same time
            if (!off && (s == 1 || nready > 0)) off = wait(&turn[s], nready - 1 + s);
            if (off) break;
            tc_fence_after();
            if (elect_one()) issue_values<0>(tO, tS, v, steps, id_o, j > 0);
            __syncwarp();
            off = wait(&p_ready[s][1], nready++);
            if (off) break;
          }
          tc_fence_after();
          if (elect_one()) {
            if (any) {
              issue_values<1>(tO, tS, v, steps, id_o, true);
              umma_commit(&empty[sv]);
              if (!more) umma_commit(&o_full[s]);
            }
            if (more) {
              issue_scores<DP>(tS, q, k, nd, idesc_bf16(SLOT, KT));
              umma_commit(&s_full[s]);
              umma_commit(&empty[sk]);
            }
            if (any) mbar_arrive(&turn[s ^ 1]);
          }
          __syncwarp();
        }
        u += n;
      }
      if (elect_one()) umma_commit(&done);
      mbar_drain(&done, 0);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int s = warp >> 2, w = warp & 3, r = tid & (SLOT - 1);
    const uint32_t lanes = static_cast<uint32_t>(w * 32) << 16;
    const uint32_t tS = tmem + s * 128 + lanes, tO = tmem + 256 + s * 128 + lanes;
    int nS = 0, nf = 0;
    // the slot's rows of the fragment that begins with a unit
    auto frag_at = [&](int u, Frag& f) {
      const int item = u / kP;
      f.prefix = 1;
      f.h = item / nPT;
      f.b = 0;
      f.k0 = u - item * kP;
      f.n = min(kP - f.k0, range.y - u);
      f.row0 = (item - f.h * nPT) * PAIR_ROWS;
      f.rows = min(PAIR_ROWS, R - f.row0);
      f.slot = item + blockIdx.x;
      f.whole = 0;                                 // (see the end of a fragment)
      f.len = a.P;
    };
    auto fetched = [&]() {
      rows_fetched();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[s]);
    };
    Frag f;
    Row x{-1, 0, nullptr};
    if (u < range.y) {
      frag_at(u, f);
      x = find_row(a, f, s * SLOT + r);
      fetch_queries<DP>(x.q, a.D, sQ + s * TILE, 32 * w);
      fetched();
    }
    while (u < range.y) {
      const bool mine = s * SLOT + r < f.rows, live = __any_sync(FULL_MASK, mine);
      float m = -INFINITY, l = 0.f;
      auto ready = [&](int half) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[s][half]);
      };
      for (int j = 0; j < f.n; ++j) {
        off = wait(&s_full[s], nS++);
        if (off) break;
        tc_fence_after();
        if (live) row_weights<Weight>(tS, tO, a.D, a.P - (f.k0 + j) * KT, a.sl2, j == 0, m, l, [&]() { ready(0); });
        else ready(0);
        ready(1);
      }
      if (off) break;
      // the next fragment's queries, behind the last products: the scores that read this one's are there
      const Frag g = f;
      const Row y = x;
      u += f.n;
      if (u < range.y) {
        frag_at(u, f);
        x = find_row(a, f, s * SLOT + r);
        fetch_queries<DP>(x.q, a.D, sQ + s * TILE, 32 * w);
      }
      off = wait(&o_full[s], nf++);
      if (off) break;
      tc_fence_after();
      if (u < range.y) fetched();
      if (live) {
        const int per = min(PAIR_ROWS, R);
        Parts own{};
        bool part = g.n < kP;
        if (!part) {                               // all of the prefix: the own entries' parts join here
          wait_for_previous();
          const Plan plan(a, a.cum[a.B], 1);         // (the prefix's units are not filled up)
          Divisor by_share;
          by_share.set(plan.share_o);
          if (mine) own = own_parts(a, plan, by_share, a.cum, g.h, g.row0 + s * SLOT + r);
          part = own.n > JOIN_PARTS;
        }
        store_rows<true>(a, tO, y, mine, m, l, part ? a.part_p + part_at(g.slot, per, a.D, s * SLOT + r, 0) : nullptr,
                         a.ml_p + (long long)g.slot * per + s * SLOT + r, per, stage + warp * STAGE_BYTES, own);
      }
      tc_fence_before();
    }
    rows_fetched();                                // (nor queries, where a wait gave up)
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
  if (tid == 0) a.errs[blockIdx.x] = aborted ? BRISK_ERR_TIMEOUT : BRISK_OK;
  // the join of what is left reads the other kernel's parts, and waits for this one alone
  wait_for_previous();
}

// ---------------------------------------------------------------- a slot a CTA
constexpr int SLOT_THREADS = SLOT + 64;            // and a copying and an issuing warp
template <int DP>
struct SlotShape {
  static constexpr int TILE = KT * DP * 2;
  static constexpr int STAGES = DP == 128 ? 2 : 4; // key and value tiles in turn
  static constexpr int SMEM = 1024 + (1 + STAGES) * TILE + 4 * STAGE_BYTES;
};

template <int DP>
__global__ void __launch_bounds__(SLOT_THREADS, 2)
attend_slot_kernel(const __grid_constant__ AttendMaps maps, const __grid_constant__ AttendArgs a) {
  constexpr int STAGES = SlotShape<DP>::STAGES, TILE = SlotShape<DP>::TILE;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* sQ = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t *ring = sQ + TILE, *stage = ring + STAGES * TILE;
  __shared__ uint64_t full[STAGES], empty[STAGES], s_full, p_ready[2], o_full, q_full, info_full[4], info_empty[4], done;
  __shared__ Frag info[4];
  __shared__ uint32_t tmem_slot;
  __shared__ Start start;
  __shared__ int aborted, bad, warp_sum[SLOT_THREADS / 32], low_of[2][4], odd_of[2][4];
  volatile int* abort_flag = &aborted;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&p_ready[s], 4);                   // the slot's warps, for either half of the keys
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(&info_full[s], 1);
      mbar_init(&info_empty[s], 4);
    }
    mbar_init(&s_full, 1);
    mbar_init(&o_full, 1);
    mbar_init(&q_full, 4);
    mbar_init(&done, 1);
    aborted = 0;
    bad = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 0) tmem_alloc(&tmem_slot, 256);      // S | O
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  let_next_begin();
  const uint32_t tmem = tmem_slot;
  auto wait = [&](uint64_t* bar, int phase) { return warp_wait(bar, phase, abort_flag, a.wait_limit); };

  const Plan plan = make_plan<SLOT_THREADS>(a, blockIdx.x, blockIdx.x == 0 ? a.cum : nullptr, warp_sum, &bad, &start);
  const int2 range = units_of(blockIdx.x, plan.share_o, plan.own0 + plan.UO);
  const bool some = range.x < range.y;
  int unit = 0, nf = 0;                            // tiles and fragments before
  bool off = false;

  if (warp == 4) {
    // copies, key and value tiles in turn, and the fragments for the others: each a fragment before its tiles
    Walk walk(a, plan, blockIdx.x, start);
    Frag f, ahead;
    unsigned cur = 0;
    bool more = walk.next(a, plan, ahead);
    auto publish = [&](int k) {
      off = k >= 4 && wait(&info_empty[k & 3], (k >> 2) - 1);
      if (!off && lane == 0) {
        info[k & 3] = ahead;
        mbar_arrive(&info_full[k & 3]);
      }
      __syncwarp();
    };
    if (more) publish(0);
    for (; !off && more; ++nf) {
      f = ahead;
      more = walk.next(a, plan, ahead);
      if (more) publish(nf + 1);
      if (off) break;
      const CUtensorMap* mk = f.prefix ? &maps.k2 : &maps.k;
      const CUtensorMap* mv = f.prefix ? &maps.v2 : &maps.v;
      for (int i = 0; i < 2 * f.n; ++i, ++cur) {
        const unsigned st = cur % STAGES;
        off = cur >= STAGES && wait(&empty[st], cur / STAGES - 1);
        if (off) break;
        if (elect_one()) load_tile<DP>(ring + st * TILE, i & 1 ? mv : mk, &full[st], f.h, (f.k0 + (i >> 1)) * KT, f.b);
        __syncwarp();
      }
    }
    // (whoever reads the tiles may have given up: none is on its way when the CTA ends)
    for (unsigned p = cur > STAGES ? cur - STAGES : 0; p < cur; ++p) mbar_drain(&full[p % STAGES], (p / STAGES) & 1);
  } else if (warp == 5) {
    const int nd = (a.D + 15) / 16;                // 16 columns a step of Q K^T, and a unit of O's width
    const uint32_t id_o = idesc_bf16(SLOT, 16 * nd) | IDESC_B_MN;
    const uint32_t q = sw128_lo(su32(sQ)), k_lo = sw128_lo(su32(ring)), v_lo = sw128_lo_mn(su32(ring), PANEL);
    const uint32_t tS = tmem, tO = tmem + 128;
    unsigned cur = 0;
    for (bool more = some; more && !off;) {
      const int fs = nf & 3;
      off = wait(&q_full, nf++);                   // (info_full came before it)
      if (off) break;
      const int n = info[fs].n, k0 = info[fs].k0, len = info[fs].len;
      more = !info[fs].last;
      for (int j = 0; j < n && !off; ++j, ++unit) {
        const unsigned sk = cur % STAGES, sv = (cur + 1) % STAGES;
        off = wait(&full[sk], cur / STAGES);
        if (off) break;
        tc_fence_after();
        if (elect_one()) {
          issue_scores<DP>(tS, q, k_lo + sk * (TILE >> 4), nd, idesc_bf16(SLOT, KT));
          umma_commit(&s_full);
          umma_commit(&empty[sk]);
        }
        __syncwarp();
        const uint32_t v = v_lo + sv * (TILE >> 4);
        const int steps = (len - (k0 + j) * KT + 15) / 16;
        off = wait(&full[sv], (cur + 1) / STAGES) || wait(&p_ready[0], unit);
        if (off) break;
        tc_fence_after();
        if (elect_one()) issue_values<0>(tO, tS, v, steps, id_o, j > 0);
        __syncwarp();
        off = wait(&p_ready[1], unit);
        if (off) break;
        tc_fence_after();
        if (elect_one()) {
          issue_values<1>(tO, tS, v, steps, id_o, true);
          umma_commit(&empty[sv]);
          if (j + 1 == n) umma_commit(&o_full);
        }
        __syncwarp();
        cur += 2;
      }
    }
    if (elect_one()) umma_commit(&done);
    mbar_drain(&done, 0);
  } else {
    const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
    const uint32_t tS = tmem + lanes, tO = tmem + 128 + lanes;
    // One turn: the next fragment's rows, this one's tiles, the next one's queries (once the scores that read
    // this one's are there), this one's end. The first turn has no fragment yet, the last no next one.
    Row y{-1, 0, nullptr};
    Frag f{};
    bool have = false, next = some;
    for (;; ++nf) {                                // this fragment is number nf - 1
      Row x{-1, 0, nullptr};
      if (next) {
        off = wait(&info_full[nf & 3], nf >> 2);
        if (off) break;
        x = find_row(a, info[nf & 3], tid);
      }
      const int fs = (nf - 1) & 1;
      const bool mine = have && tid < f.rows, live = __any_sync(FULL_MASK, mine);
      float m = -INFINITY, l = 0.f;
      int low = f.len;                             // entries from here on are hidden from some row
      if (have) {
#pragma unroll
        for (int w = 0; w < 4; ++w) low = min(low, low_of[fs][w]);
        auto ready = [&](int half) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_ready[half]);
        };
        for (int j = 0; j < f.n; ++j, ++unit) {
          const int t0 = (f.k0 + j) * KT, end = min(f.len - t0, KT);   // entries in use of the tile
          // values that some row does not see, and those behind the last entry that the last step reads
          const int v0 = max(low - t0, 0), v1 = min((end + 15) & ~15, KT);
          const bool clean = !f.prefix && v0 < v1;   // (behind the prefix's last entry there are zeros)
          off = wait(&s_full, unit);
          if (off) break;
          tc_fence_after();
          if (live)
            row_weights<Weight>(tS, tO, a.D, mine ? y.lim - t0 : KT, a.sl2, j == 0, m, l,
                        [&]() { if (!clean) ready(0); });
          if (clean) {
            const unsigned pl = 2 * unit + 1, st = pl % STAGES;
            off = wait(&full[st], pl / STAGES);
            if (off) break;
            const bool odd = clean_values<DP>(ring + st * TILE, v0, v1, end, tid);
            if (__any_sync(FULL_MASK, odd) && lane == 0) odd_of[fs][warp] = 1;
          }
          if (clean || !live) ready(0);
          ready(1);
        }
        if (off) break;
      }
      if (next) fetch_queries<DP>(x.q, a.D, sQ, 32 * warp);
      if (have) {
        off = wait(&o_full, nf - 1);
        if (off) break;
        tc_fence_after();
      }
      if (next) {
        const int low_next = __reduce_min_sync(FULL_MASK, x.id >= 0 ? x.lim : info[nf & 3].len);
        if (lane == 0) {
          low_of[nf & 1][warp] = low_next;
          odd_of[nf & 1][warp] = 0;
        }
        rows_fetched();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_full);
      }
      if (have) {
        if (live) {
          const int per = min(SLOT, f.prefix ? plan.R : plan.LG);
          float* part = f.whole ? nullptr : (f.prefix ? a.part_p : a.part_o) + part_at(f.slot, per, a.D, tid, 0);
          store_rows<false>(a, tO, y, mine, m, l, part, (f.prefix ? a.ml_p : a.ml_o) + (long long)f.slot * per + tid, per,
                            stage + warp * STAGE_BYTES, Parts{});
          __syncwarp();
          // (the warps' words of this fragment were written before the products that o_full tells of, and other
          // lanes may have stored this row)
          if (!f.prefix && low < f.len && (odd_of[fs][0] | odd_of[fs][1] | odd_of[fs][2] | odd_of[fs][3]) && mine && y.id >= 0)
            add_odd(a, f.b, f.h, max(low, f.k0 * KT), min(y.lim, (f.k0 + f.n) * KT), part, per,
                    static_cast<__nv_bfloat16*>(a.out) + (long long)y.id * a.D);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&info_empty[(nf - 1) & 3]);
      }
      if (!next) break;
      off = wait(&q_full, nf);
      if (off) break;
      f = info[nf & 3];
      y = x;
      have = true;
      next = !f.last;
    }
    rows_fetched();                                // (queries, where a wait gave up)
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 256);
  if (tid == 0)
    a.errs[a.sh.grid_p + blockIdx.x] =
        aborted ? BRISK_ERR_TIMEOUT : (bad && blockIdx.x == 0 ? BRISK_ERR_INVALID_ARG : BRISK_OK);
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
  cuuint32_t box[4] = {64, 1, TC_KT, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(v.p), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_prefix_tc(const AttendArgs& a, cudaStream_t stream) {
  AttendMaps maps;
  if (!make_cache_map(&maps.k, a.kp, a.D, a.Hkv, a.P, 1) || !make_cache_map(&maps.v, a.vp, a.D, a.Hkv, a.P, 1))
    return cudaErrorInvalidValue;
  maps.k2 = maps.k;
  maps.v2 = maps.v;
  auto pair = a.D > 64 ? attend_pair_kernel<128> : attend_pair_kernel<64>;
  const size_t smem = a.D > 64 ? PairShape<128>::SMEM : PairShape<64>::SMEM;
  cudaError_t e = set_up_kernel(pair, CARVEOUT_FULL_KB, smem);
  return e != cudaSuccess ? e : launch_early(pair, a.sh.grid_p, PAIR_THREADS, smem, stream, true, maps, a);
}

cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t stream) {
  AttendMaps maps;
  if (!make_cache_map(&maps.k2, a.kp, a.D, a.Hkv, a.P, 1) || !make_cache_map(&maps.v2, a.vp, a.D, a.Hkv, a.P, 1) ||
      !make_cache_map(&maps.k, a.ko, a.D, a.Hkv, a.S, a.B) || !make_cache_map(&maps.v, a.vo, a.D, a.Hkv, a.S, a.B))
    return cudaErrorInvalidValue;
  auto slot = a.D > 64 ? attend_slot_kernel<128> : attend_slot_kernel<64>;
  const size_t slot_smem = a.D > 64 ? SlotShape<128>::SMEM : SlotShape<64>::SMEM;
  cudaError_t e = set_up_kernel(slot, CARVEOUT_FULL_KB, slot_smem);
  if (e == cudaSuccess) e = launch_early(slot, a.sh.grid_o, SLOT_THREADS, slot_smem, stream, false, maps, a);
  if (e == cudaSuccess && a.sh.grid_p > 0) e = launch_prefix_tc(a, stream);
  return e;
}

}  // namespace brisk
