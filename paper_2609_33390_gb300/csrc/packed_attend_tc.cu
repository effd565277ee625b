// Attention over own caches in 4 bits on the tensor cores of sm_103a, for many query rows a key head.
//
// As attend_slot_kernel (cache_attend_tc.cu), a slot of 128 query rows a CTA, two CTAs an SM, but the tiles of keys and
// values are not copied: three warps for each read their codes to registers and write them as fp16, in which they are
// exact, where the products take them from shared memory. The queries become fp16 too (both operands of a product
// have one type), each row scaled by a power of two so that its largest magnitude is 2^14 to 2^15: exact from 2^-31 of it
// on, below off by up to 2^-39 of it. (Keys as bf16 instead cost more, in every tile, than the queries' change once a
// fragment: 217 and 197 us, 128 blocks.) Weights are fp16, taken relative to 2^-10 of the held maximum: off by 2^-11 of
// themselves, or 2^-35 of the maximum. Scores are taken 64 keys at a time, in two places of TMEM, so that the tensor cores work on the next while a slot's threads take exponentials. Codes that a row
// does not see stand for finite numbers, and rows of a tile behind the last entry are written as zeros.
//
// Bound by a unit's chain (codes, tiles, scores, exponentials, values) with two CTAs an SM to overlap: 128 blocks of 32
// positions, 32 heads on 8, D = 128, over 512 to 2048 own entries each 121 us, where the products alone would take 45.
// Tensor cores are active 26 % of the time, 48 % of the issue slots are used; a fragment's ends (its queries' change, its
// parts) take about as long as three of its units of 128 keys.
// Codes copied to shared memory first (cp.async) took 275 us of the whole call, where reading them to registers took 260.
#include "attend_tc.cuh"
#include "packed.cuh"

namespace brisk {
namespace {

using Weight = WeightAs<__half>;
constexpr int CODE_WARPS = 3;                      // that read the codes of keys, and as many for values
constexpr int THREADS = SLOT + 64 + 64 * CODE_WARPS;   // a planning and an issuing warp, and those that read codes
constexpr int HALF = 64;                           // keys of a step: half a unit
constexpr int HALF_PANEL = HALF * 128;             // bytes of a panel of its 64 columns
template <int DP>
struct Shape4 {
  static constexpr int TILE = HALF * DP * 2;
  static constexpr int STAGES = DP == 128 ? 4 : 8; // key and value tiles in turn
  static constexpr int SMEM = 1024 + 2 * TILE + STAGES * TILE + 4 * STAGE_BYTES;
};

// The part of a tile of codes that a warp reads: a lane has 16 bytes, 32 channels, of a row of each group of 8 (16, up to
// 64 channels), so that eight neighbouring lanes write eight rows, whose pieces are swizzled into different banks. Warp
// w of the CODE_WARPS has groups w, w + CODE_WARPS, ...
template <int DP>
struct Codes {
  static constexpr int PIECES = DP / 32, ROWS = 32 / PIECES, GROUPS = HALF / ROWS, N = (GROUPS + CODE_WARPS - 1) / CODE_WARPS;
  static constexpr int STEP = CODE_WARPS * ROWS;   // rows between a lane's groups
  uint32_t w[N][4], s[N];
  const uint8_t *codes, *scales;                   // of the lane's first row of the next tile
  int left;                                        // rows from that one on (none: channels that are not there)
  static __device__ __forceinline__ int row() { return (threadIdx.x & 7) | (PIECES == 2 ? (threadIdx.x >> 1 & 8) : 0); }
  static __device__ __forceinline__ int piece() { return PIECES == 2 ? threadIdx.x >> 3 & 1 : threadIdx.x >> 3 & 3; }

  __device__ __forceinline__ void begin(const PackedView& v, const Frag& f, int cw, int D) {
    const int first = f.k0 * KT + cw * ROWS + row();
    codes = v.codes + f.b * v.seq + f.h * v.head + (unsigned long long)(uint32_t)first * v.tok + 16 * piece();
    scales = v.scales + f.b * v.sseq + f.h * v.shead + (unsigned long long)(uint32_t)first * v.stok + 2 * piece();
    left = 32 * piece() < D ? f.len - first : -(1 << 30);
  }
  // (zeros where there is nothing to read)
  __device__ __forceinline__ void read(int i, uint32_t tok, uint32_t stok, int cw, int D) {
    const bool wide = (D & 31) == 0, full = 32 * piece() + 16 < D;   // (else rows start on 8 bytes)
    {
      w[i][0] = w[i][1] = w[i][2] = w[i][3] = 0;
      s[i] = 0;
      if (STEP * i < left && (i + 1 < N || cw + i * CODE_WARPS < GROUPS)) {
        const uint8_t* p = codes + (unsigned long long)(STEP * i) * tok;
        if (wide) {
          const uint4 z = __ldg(reinterpret_cast<const uint4*>(p));
          w[i][0] = z.x; w[i][1] = z.y; w[i][2] = z.z; w[i][3] = z.w;
        } else {
          const uint2 z = __ldg(reinterpret_cast<const uint2*>(p));
          w[i][0] = z.x; w[i][1] = z.y;
          if (full) {
            const uint2 z8 = __ldg(reinterpret_cast<const uint2*>(p + 8));
            w[i][2] = z8.x; w[i][3] = z8.y;
          }
        }
        s[i] = __ldg(reinterpret_cast<const uint16_t*>(scales + (unsigned long long)(STEP * i) * stok));
      }
    }
  }
  __device__ __forceinline__ void go_on(uint32_t tok, uint32_t stok) {
    codes += (unsigned long long)HALF * tok;
    scales += (unsigned long long)HALF * stok;
    left -= HALF;
  }
  // Where the lane's words of its first row go in a tile: they differ in the bits that the swizzle changes.
  static __device__ __forceinline__ void places(int (&at)[4], int cw) {
    const int first = (piece() >> 1) * HALF_PANEL + (cw * ROWS + row()) * 128 + (((piece() & 1) * 4 ^ (row() & 7)) << 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      at[k] = first ^ k << 4;
      asm volatile("" : "+r"(at[k]));              // (or they would be worked out again for every store)
    }
  }
  __device__ __forceinline__ void write(int i, uint8_t* tile, const int (&at)[4], int cw) const {
    if (i + 1 < N || cw + i * CODE_WARPS < GROUPS) {
      const uint32_t by[2] = {scale_f16(s[i] & 255), scale_f16(s[i] >> 8)};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t h[4];
        from_codes(w[i][k], h);
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = mul_f16(h[j], by[k >> 1]);
        *reinterpret_cast<uint4*>(tile + at[k] + STEP * i * 128) = make_uint4(h[0], h[1], h[2], h[3]);
      }
    }
  }
};

// A row of queries, as fetch_queries left it, becomes fp16 in its place; what its scores are to be multiplied by. (Four
// pieces are read at once: one after the other took 6000 cycles, a tenth of the kernel's time. No more, since this runs
// once a fragment and its instructions have to be fetched.)
template <int DP>
__device__ __forceinline__ float scale_query(uint8_t* tile, int row, int D, float sl2) {
  uint8_t* at = tile + row * 128;
  auto piece = [&](int c) { return reinterpret_cast<uint4*>(at + (c >> 3) * PANEL + (((c ^ row) & 7) << 4)); };
  uint32_t top = 0;                                // of both halves' 16 bits: magnitudes compare as their bits do
#pragma unroll 1
  for (int c0 = 0; 8 * c0 < D; c0 += 4) {
    uint4 x[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) x[c] = *piece(c0 + c);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t t = __vmaxu2(__vmaxu2(x[c].x & 0x7fff7fffu, x[c].y & 0x7fff7fffu),
                                  __vmaxu2(x[c].z & 0x7fff7fffu, x[c].w & 0x7fff7fffu));
      if (8 * (c0 + c) < D) top = __vmaxu2(top, t);    // (behind the row's end there may be anything)
    }
  }
  const int up = query_shift(max(top << 16, top & 0xffff0000u));
  const f32x2 by = pack2(exp2_of(up), exp2_of(up));
  auto change = [&](uint32_t x) {
    float lo, hi;
    unpack2(mul2(pack2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)), by), lo, hi);
    return Weight::pair(lo, hi);
  };
#pragma unroll 1
  for (int c0 = 0; 8 * c0 < D; c0 += 4) {
    uint4 x[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) x[c] = *piece(c0 + c);
#pragma unroll
    for (int c = 0; c < 4; ++c) *piece(c0 + c) = make_uint4(change(x[c].x), change(x[c].y), change(x[c].z), change(x[c].w));
  }
  return query_scale(sl2, up);
}

// row_weights (see there) of HALF keys. before(): waits until nothing is on its way to O (false: in vain).
template <typename Before>
__device__ __forceinline__ void half_weights(uint32_t tS, uint32_t tO, int D, int seen, float sl2, bool first, float& m, float& l,
                                             Before before) {
  float s[HALF];
  tmem_ld64(tS, s);
  if (__any_sync(FULL_MASK, seen < HALF)) {
#pragma unroll
    for (int c = 0; c < HALF; ++c) s[c] = c < seen ? s[c] : -INFINITY;
  }
  float top[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
  for (int c = 4; c + 8 <= HALF; c += 8)
#pragma unroll
    for (int i = 0; i < 4; ++i) top[i] = fmaxf(fmaxf(top[i], s[c + i]), s[c + 4 + i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) top[i] = fmaxf(top[i], s[HALF - 4 + i]);
  const float t = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * sl2;
  const bool over = t > m + Weight::LAZY;
  if (__any_sync(FULL_MASK, over)) {
    const float alpha = over ? ex2(m - t) : 1.f;   // (t is no -inf)
    if (over) m = t;
    l *= alpha;
    if (!first && before())
#pragma unroll 1
      for (int c = 0; c < D; c += 16) {
        float o[16];
        tmem_ld16(tO + c, o);
        uint32_t x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(o[i] * alpha);
        tmem_st16(tO + c, x);
      }
  }
  const float ms = m == -INFINITY ? 0.f : m - Weight::SHIFT;
  const f32x2 scale2 = pack2(sl2, sl2), minus2 = pack2(-ms, -ms);
  f32x2 sum0 = pack2(0.f, 0.f), sum1 = sum0;
#pragma unroll
  for (int c0 = 0; c0 < HALF; c0 += 32) {
    uint32_t p[16];
#pragma unroll
    for (int c = 0; c < 32; c += 4) {
      float x[4];
      unpack2(fma2(pack2(s[c0 + c], s[c0 + c + 1]), scale2, minus2), x[0], x[1]);
      unpack2(fma2(pack2(s[c0 + c + 2], s[c0 + c + 3]), scale2, minus2), x[2], x[3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = ex2(x[i]);
      sum0 = add2(sum0, pack2(x[0], x[1]));
      sum1 = add2(sum1, pack2(x[2], x[3]));
      p[c / 2] = Weight::pair(x[0], x[1]);
      p[c / 2 + 1] = Weight::pair(x[2], x[3]);
    }
    tmem_st16(tS + c0 / 2, p);
  }
  float x[2];
  unpack2(add2(sum0, sum1), x[0], x[1]);
  l += x[0] + x[1];
  tmem_st_wait();
}

// The steps of a fragment that have entries.
__device__ __forceinline__ int halves_of(const Frag& f) { return (min(f.len - f.k0 * KT, f.n * KT) + HALF - 1) / HALF; }

// The products of a slot with a half of a tile: scores, and values for `steps` <= 4 steps of 16 keys.
template <int DP>
__device__ __forceinline__ void issue_half_scores(uint32_t tS, uint32_t q_lo, uint32_t k_lo, int nd, uint32_t idesc) {
#pragma unroll
  for (int kk = 0; kk < DP / 16; ++kk) {
    const uint32_t o = 2 * (kk & 3);
    if (kk < nd) umma(tS, sw128(q_lo + (kk >> 2) * (PANEL >> 4) + o), sw128(k_lo + (kk >> 2) * (HALF_PANEL >> 4) + o), idesc, kk > 0);
  }
}
__device__ __forceinline__ void issue_half_values(uint32_t tO, uint32_t tP, uint32_t v_lo, int steps, uint32_t idesc, bool begun) {
#pragma unroll
  for (int kk = 0; kk < HALF / 16; ++kk)
    if (kk < steps) umma_ts(tO, tP + 8 * kk, sw128(v_lo + kk * 128), idesc, begun || kk > 0);
}

template <int DP>
__global__ void __launch_bounds__(THREADS, 2)
packed_slot_kernel(const __grid_constant__ PackedArgs p) {
  constexpr int STAGES = Shape4<DP>::STAGES, TILE = Shape4<DP>::TILE;
  const AttendArgs& a = p.a;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* sQ = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t *ring = sQ + 2 * TILE, *stage = ring + STAGES * TILE;
  __shared__ uint64_t full[STAGES], empty[STAGES], s_full[2], p_ready[2], v_done[2], o_full, q_full, info_full[4], info_empty[4], done;
  __shared__ Frag info[4];
  __shared__ uint32_t tmem_slot;
  __shared__ Start start;
  __shared__ Plan plan;
  __shared__ Walk walk;
  __shared__ int aborted, bad, warp_sum[THREADS / 32];
  volatile int* abort_flag = &aborted;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], CODE_WARPS);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&s_full[s], 1);
      mbar_init(&p_ready[s], 4);                   // the slot's warps
      mbar_init(&v_done[s], 1);
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(&info_full[s], 1);
      mbar_init(&info_empty[s], 4 + 2 * CODE_WARPS);
    }
    mbar_init(&o_full, 1);
    mbar_init(&q_full, 4);
    mbar_init(&done, 1);
    aborted = 0;
    bad = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 0) tmem_alloc(&tmem_slot, 256);      // S of two halves | O
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  let_next_begin();
  const uint32_t tmem = tmem_slot;
  auto wait = [&](uint64_t* bar, int phase) { return warp_wait(bar, phase, abort_flag, a.wait_limit); };

  // (the plan and the walk through it in shared memory: the others need their registers)
  {
    const Plan made = make_plan<THREADS>(a, blockIdx.x, blockIdx.x == 0 ? a.cum : nullptr, warp_sum, &bad, &start);
    if (tid == 0) {
      plan = made;
      walk = Walk(a, made, blockIdx.x, start);
    }
  }
  __syncthreads();
  const bool some = walk.u < walk.end;
  __syncthreads();                                 // (before it moves)
  int half = 0, nf = 0;                            // halves of tiles and fragments before
  bool off = false;

  // (384 threads of 80 registers: 128 x 112 and 256 x 64)
  if (warp >= 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == 4) {
      // the fragments, each published while the one before is worked on
      for (bool more = some; more && !off; ++nf) {
        off = nf >= 4 && wait(&info_empty[nf & 3], (nf >> 2) - 1);
        int last = 1;
        if (!off && lane == 0) {
          walk.next(a, plan, info[nf & 3]);
          last = info[nf & 3].last;
          mbar_arrive(&info_full[nf & 3]);
        }
        more = __shfl_sync(FULL_MASK, last, 0) == 0;
      }
    } else if (warp == 5) {
      const int nd = a.D / 16;                     // steps of 16 columns of Q K^T, and units of O's width
      const uint32_t id_s = idesc_f16(SLOT, HALF), id_o = idesc_f16(SLOT, 16 * nd) | IDESC_B_MN;
      const uint32_t q = sw128_lo(su32(sQ)), k_lo = sw128_lo(su32(ring)), v_lo = sw128_lo_mn(su32(ring), HALF_PANEL);
      for (bool more = some; more && !off;) {
        const int fs = nf & 3;
        off = wait(&q_full, nf++);                 // (info_full came before it)
        if (off) break;
        const int n = halves_of(info[fs]), len = info[fs].len - info[fs].k0 * KT;
        more = !info[fs].last;
        // The scores of a step come two steps ahead of its values: while the slot's threads take one step's weights, the
        // products with the values of the one before and the scores of the one behind run.
        auto scores = [&](int h) {
          const unsigned cur = 2 * (half + h), st = cur % STAGES;
          off = wait(&full[st], cur / STAGES);
          if (off) return;
          fence_async_smem();
          tc_fence_after();
          if (elect_one()) {
            issue_half_scores<DP>(tmem + ((half + h) & 1) * HALF, q, k_lo + st * (TILE >> 4), nd, id_s);
            umma_commit(&s_full[(half + h) & 1]);
            umma_commit(&empty[st]);
          }
          __syncwarp();
        };
        scores(0);
        if (n > 1 && !off) scores(1);
        for (int h = 0; h < n && !off; ++h) {
          const unsigned cur = 2 * (half + h) + 1, st = cur % STAGES;
          off = wait(&full[st], cur / STAGES) || wait(&p_ready[(half + h) & 1], (half + h) >> 1);
          if (off) break;
          fence_async_smem();
          tc_fence_after();
          if (elect_one()) {
            issue_half_values(tmem + 2 * HALF, tmem + ((half + h) & 1) * HALF, v_lo + st * (TILE >> 4),
                              (len - h * HALF + 15) / 16, id_o, h > 0);
            umma_commit(&v_done[(half + h) & 1]);
            umma_commit(&empty[st]);
            if (h + 1 == n) umma_commit(&o_full);
          }
          __syncwarp();
          if (h + 2 < n) scores(h + 2);
        }
        half += n;
      }
      if (elect_one()) umma_commit(&done);
      mbar_drain(&done, 0);
    } else if (some) {
      // codes to fp16, keys or values; a step's are on their way to registers while the one before is written
      const int value = warp - 6 >= CODE_WARPS, cw = warp - 6 - value * CODE_WARPS;
      const uint32_t tok = value ? p.v.tok : p.k.tok, stok = value ? p.v.stok : p.k.stok;
      constexpr int N = Codes<DP>::N;
      Codes<DP> x;
      int at[4];
      Codes<DP>::places(at, cw);
      int left = 0, last = 0;                      // steps of the fragment that are not read yet
      auto next = [&]() {                          // whether there is another step to read
        if (left == 0 && !last) {
          off = wait(&info_full[nf & 3], nf >> 2);
          if (off) return false;
          const Frag& f = info[nf & 3];
          left = halves_of(f);
          last = f.last;
          if (value) x.begin(p.v, f, cw, a.D);
          else x.begin(p.k, f, cw, a.D);
          __syncwarp();
          if (lane == 0) mbar_arrive(&info_empty[nf & 3]);
          ++nf;
        }
        return left > 0;
      };
      bool more = next();
      if (more) {
#pragma unroll
        for (int i = 0; i < N; ++i) x.read(i, tok, stok, cw, a.D);
        x.go_on(tok, stok);
        --left;
      }
      for (unsigned cur = value; more; cur += 2) {
        const unsigned st = cur % STAGES;
        more = next();
        off = off || (cur >= STAGES && wait(&empty[st], cur / STAGES - 1));
        if (off) break;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          x.write(i, ring + st * TILE, at, cw);
          if (more) x.read(i, tok, stok, cw, a.D);
        }
        if (more) {
          x.go_on(tok, stok);
          --left;
        }
        // (the warp that issues the products fences them off: this one's fence would wait for its loads, too)
        __syncwarp();
        if (lane == 0) mbar_arrive(&full[st]);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
    const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
    const uint32_t tO = tmem + 2 * HALF + lanes;
    // One turn: the next fragment's rows, this one's tiles, the next one's queries (once the scores that read
    // this one's are there), this one's end. The first turn has no fragment yet, the last no next one.
    // (of a fragment's words only those that every tile wants stay in registers)
    int y_id = -1, y_lim = 0;                      // this fragment's row of the thread: see Row
    float y_scale = 0.f;                           // what its scores are multiplied by
    bool have = false, next = some;
    for (;; ++nf) {                                // this fragment is number nf - 1
      const Frag& f = info[(nf - 1) & 3];
      Row x{-1, 0, nullptr};
      if (next) {
        off = wait(&info_full[nf & 3], nf >> 2);
        if (off) break;
        x = find_row(a, info[nf & 3], tid);
      }
      const bool live = __any_sync(FULL_MASK, have && tid < f.rows);   // (rows of this fragment)
      float m = -INFINITY, l = 0.f;
      if (have) {
        int seen = tid < f.rows ? y_lim - f.k0 * KT : 0x3fffffff;
        const int n = halves_of(f);
        for (int h = 0; h < n; ++h, ++half, seen -= HALF) {
          off = wait(&s_full[half & 1], half >> 1);
          if (off) break;
          tc_fence_after();
          // (the last scores that read this fragment's queries are there)
          if (h + 1 == n && next) fetch_queries<DP>(x.q, a.D, sQ, 32 * warp);
          if (live)
            half_weights(tmem + (half & 1) * HALF + lanes, tO, a.D, seen, y_scale, h == 0, m, l, [&]() {
              // (the half before's products; the ones before them came before these scores. A phase that no one may have
              // waited for: the next of this barrier comes after this half's weights.)
              off = wait(&v_done[(half - 1) & 1], (half - 1) >> 1);
              tc_fence_after();
              return !off;
            });
          if (off) break;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_ready[half & 1]);
        }
        if (off) break;
      } else if (next) {
        fetch_queries<DP>(x.q, a.D, sQ, 32 * warp);
      }
      float x_scale = 0.f;
      if (next) {
        rows_fetched();
        __syncwarp();
        if (x.q) x_scale = scale_query<DP>(sQ, tid, a.D, a.sl2);
        fence_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_full);
      }
      if (have) {
        off = wait(&o_full, nf - 1);
        if (off) break;
        tc_fence_after();
        if (live) {
          const int per = min(SLOT, plan.LG);
          float* part = f.whole ? nullptr : a.part_o + part_at(f.slot, per, a.D, tid, 0);
          store_rows<false>(a, tO, Row{y_id, y_lim, nullptr}, tid < f.rows, m == -INFINITY ? m : m - Weight::SHIFT, l, part,
                            a.ml_o + (long long)f.slot * per + tid, per, stage + warp * STAGE_BYTES, Parts{});
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&info_empty[(nf - 1) & 3]);
      }
      if (!next) break;
      off = wait(&q_full, nf);
      if (off) break;
      y_id = x.id;
      y_lim = x.lim;
      y_scale = x_scale;
      have = true;
      next = !info[nf & 3].last;
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

cudaError_t launch_packed_tc(const PackedArgs& p, cudaStream_t stream) {
  auto kernel = p.a.D > 64 ? packed_slot_kernel<128> : packed_slot_kernel<64>;
  const size_t smem = p.a.D > 64 ? Shape4<128>::SMEM : Shape4<64>::SMEM;
  cudaError_t e = set_up_kernel(kernel, CARVEOUT_FULL_KB, smem);
  return e != cudaSuccess ? e : launch_early(kernel, p.a.sh.grid_o, THREADS, smem, stream, false, p);
}

}  // namespace brisk
