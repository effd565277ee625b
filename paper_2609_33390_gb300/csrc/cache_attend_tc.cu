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
constexpr int ATT_THREADS = SOFT_THREADS + 64;     // and a copying and an issuing warp
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

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y,
                                            int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(su32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(su32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(su32(bar)) : "memory");
}
// The barrier of the two slots' warps.
__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

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

template <int DP>
__global__ void __launch_bounds__(ATT_THREADS, 1)
attend_tc_kernel(const __grid_constant__ AttendMaps maps, const __grid_constant__ AttendArgs a) {
  using Sh = Shape<DP>;
  constexpr int STAGES = Sh::STAGES, TILE = Sh::TILE;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = base;                              // [2][DP / 64][128 rows][128 B], swizzled
  uint8_t* ring = base + 2 * TILE;
  int32_t* cum = reinterpret_cast<int32_t*>(ring + STAGES * TILE);
  __shared__ uint64_t full[STAGES], empty[STAGES], s_full[2], p_ready[2], o_full[2], q_full, done;
  __shared__ uint32_t tmem_slot;
  __shared__ int aborted, bad, warp_sum[ATT_THREADS / 32], low_of[8], odd_of[8];
  __shared__ float2 ml_of[2][SLOT];
  volatile int* abort_flag = &aborted;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&s_full[s], 1);
      mbar_init(&p_ready[s], 4);                   // a lane of each of the slot's warps
      mbar_init(&o_full[s], 1);
    }
    mbar_init(&q_full, 1);
    mbar_init(&done, 1);
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

  auto wait = [&](uint64_t* bar, int phase) {
    if (*abort_flag) return false;
    if (mbar_wait(bar, phase & 1, abort_flag, a.wait_limit)) return true;
    *abort_flag = 1;
    return false;
  };
  Walk walk(plan, cum, blockIdx.x);
  Frag f;
  int pos = 0;                                     // ring places of the fragments before this one

  if (warp == 8) {
    if (lane == 0) {
      // copies: a key or value tile at a time, in the ring's order
      int issued = 0;
      while (walk.next(plan, cum, f)) {
        const bool pair = f.rows > SLOT;
        const CUtensorMap* mk = f.prefix ? &maps.kp : &maps.ko;
        const CUtensorMap* mv = f.prefix ? &maps.vp : &maps.vo;
        int nk = 0, nvt = 0;
        for (int i = 0; i < 2 * f.n; ++i) {
          const bool key = nk < f.n && k_place(pair, nk) == i;
          const int t0 = (f.k0 + (key ? nk++ : nvt++)) * KT, p = pos + i, st = p % STAGES;
          if (p >= STAGES) wait(&empty[st], p / STAGES - 1);
          if (*abort_flag) break;
          mbar_expect_tx(&full[st], TILE);
          for (int c = 0; c < DP / 64; ++c)
            tma_load_4d(ring + st * TILE + c * PANEL, key ? mk : mv, &full[st], c * 64, f.h, t0, f.b);
          issued = p + 1;
        }
        pos += 2 * f.n;
      }
      if (*abort_flag)
        for (int p = issued > STAGES ? issued - STAGES : 0; p < issued; ++p)
          mbar_drain(&full[p % STAGES], (p / STAGES) & 1);
    }
  } else if (warp == 9) {
    if (lane == 0) {
      // products
      const int nd = (a.D + 15) / 16;              // 16 columns a step of Q K^T, and a unit of O's width
      const uint32_t id_s = idesc_bf16(SLOT, KT), id_o = idesc_bf16(SLOT, 16 * nd) | IDESC_B_MN;
      int nfrag = 0, nready[2] = {0, 0};
      auto scores = [&](int s, int qslot, int st) {
        if (*abort_flag) return;
        const uint32_t qa = su32(sQ + qslot * TILE), ka = su32(ring + st * TILE);
        for (int kk = 0; kk < nd; ++kk) {
          const uint64_t off = (kk >> 2) * (PANEL >> 4) + 2 * (kk & 3);
          umma(tmem + s * 128, sw128_desc(qa) + off, sw128_desc(ka) + off, id_s, kk > 0);
        }
        umma_commit(&s_full[s]);
      };
      while (walk.next(plan, cum, f)) {
        const bool pair = f.rows > SLOT;
        const int end = f.prefix ? a.P : clamped_len(a, f.b);
        auto stage = [&](int place) {
          const int p = pos + place;
          wait(&full[p % STAGES], p / STAGES);
          return p % STAGES;
        };
        auto values = [&](int s, int j, int st, bool first) {
          wait(&p_ready[s], nready[s]++);
          if (*abort_flag) return;
          tc_fence_after();
          const int keys = min(KT, end - (f.k0 + j) * KT);
          const uint64_t vd = sw128_desc_mn(su32(ring + st * TILE), PANEL);
          for (int kk = 0; kk < (keys + 15) / 16; ++kk)
            umma_ts(tmem + 256 + s * 128, tmem + s * 128 + 8 * kk, vd + kk * 128, id_o, !first || kk > 0);
        };
        auto release = [&](int st) { if (!*abort_flag) umma_commit(&empty[st]); };
        wait(&q_full, nfrag++);
        tc_fence_after();
        if (pair) {
          int st = stage(0);
          tc_fence_after();
          scores(0, 0, st);
          scores(1, 1, st);
          release(st);
          for (int j = 0; j < f.n; ++j) {
            const int sv = stage(v_place(true, j, f.n));
            int sk = 0;
            for (int s = 0; s < 2; ++s) {
              values(s, j, sv, j == 0);
              if (s == 1) release(sv);
              if (j + 1 < f.n) {
                if (s == 0) sk = stage(k_place(true, j + 1));
                tc_fence_after();
                scores(s, s, sk);
                if (s == 1) release(sk);
              } else if (!*abort_flag) {
                umma_commit(&o_full[s]);
              }
            }
          }
        } else {
          for (int j = 0; j < 2 && j < f.n; ++j) {
            const int st = stage(k_place(false, j));
            tc_fence_after();
            scores(j, 0, st);
            release(st);
          }
          for (int j = 0; j < f.n; ++j) {
            const int s = j & 1, sv = stage(v_place(false, j, f.n));
            values(s, j, sv, j < 2);
            release(sv);
            if (j + 2 < f.n) {
              const int sk = stage(k_place(false, j + 2));
              tc_fence_after();
              scores(s, 0, sk);
              release(sk);
            } else if (!*abort_flag) {
              umma_commit(&o_full[s]);
            }
          }
        }
        pos += 2 * f.n;
      }
      umma_commit(&done);
      mbar_drain(&done, 0);
    }
  } else {
    const int s = warp >> 2, r = tid & (SLOT - 1), D = a.D;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + s * 128 + lanes, tO = tmem + 256 + lanes;
    int nS = 0, nO = 0;                            // tiles and fragments this slot had
    while (walk.next(plan, cum, f)) {
      const bool pair = f.rows > SLOT;
      const int len = f.prefix ? a.P : clamped_len(a, f.b);
      tc_fence_before();
      soft_sync();                                 // the last fragment's Q, O and words are done with
      // Q: 16 bytes a thread, rows beyond the fragment's and columns beyond D zero
      constexpr int VPR = DP / 8;                  // 16-byte pieces of a row
      for (int e = tid; e < (pair ? 2 : 1) * SLOT * VPR; e += SOFT_THREADS) {
        const int row = e / VPR, c = e % VPR;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < f.rows && 8 * c < D) {
          int token, head;
          row_of(a, f, row, token, head);
          const int b = token / a.L, i = token - b * a.L;
          v = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.seq +
                                              i * a.q.tok + head * a.q.head + 8 * c);
        }
        const int in = row & (SLOT - 1);
        *reinterpret_cast<uint4*>(sQ + (row >> 7) * TILE + (c >> 3) * PANEL + in * 128 + ((c & 7) ^ (in & 7)) * 16) = v;
      }
      fence_async_smem();
      const int my = pair ? s * SLOT + r : r;      // this thread's row
      const bool mine = my < f.rows;
      int token = 0, head = 0, lim = 0;
      if (mine) {
        row_of(a, f, my, token, head);
        lim = row_limit(a, f, token, len);
      }
      const int warp_low = __reduce_min_sync(FULL_MASK, mine ? lim : len);
      if (lane == 0) {
        low_of[warp] = warp_low;
        odd_of[warp] = 0;
      }
      soft_sync();
      if (tid == 0) mbar_arrive(&q_full);
      int low = len;                               // entries from here on are hidden from some row
#pragma unroll
      for (int w = 0; w < 8; ++w) low = min(low, low_of[w]);
      const bool warp_live = __any_sync(FULL_MASK, mine);

      float m = -INFINITY, l = 0.f;
      int tiles = 0;
      for (int j = pair ? 0 : s; j < f.n; j += pair ? 1 : 2, ++tiles) {
        const int t0 = (f.k0 + j) * KT, end = min(len - t0, KT);   // entries in use of the tile
        wait(&s_full[s], nS++);
        __syncwarp();
        tc_fence_after();
        if (warp_live) {
          float v[KT];
          tmem_ld128(tS, v);
          if (__any_sync(FULL_MASK, mine && lim - t0 < KT)) {
            const int n = lim - t0;
#pragma unroll
            for (int c = 0; c < KT; ++c) v[c] = c < n ? v[c] : -INFINITY;
          }
          float top = v[0], top1 = v[1], top2 = v[2], top3 = v[3];
#pragma unroll
          for (int c = 4; c < KT; c += 4) {
            top = fmaxf(top, v[c]);
            top1 = fmaxf(top1, v[c + 1]);
            top2 = fmaxf(top2, v[c + 2]);
            top3 = fmaxf(top3, v[c + 3]);
          }
          const float t = fmaxf(fmaxf(top, top1), fmaxf(top2, top3)) * a.sl2;
          if (__any_sync(FULL_MASK, t > m + LAZY)) {
            const float mn = fmaxf(m, t), alpha = ex2(m - (mn == -INFINITY ? 0.f : mn));
            m = mn;
            l *= alpha;
            if (tiles > 0)
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
          float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
          for (int c0 = 0; c0 < KT; c0 += 32) {
            uint32_t p[16];
#pragma unroll
            for (int c = 0; c < 32; c += 2) {
              const float p0 = ex2(fmaf(v[c0 + c], a.sl2, -ms)), p1 = ex2(fmaf(v[c0 + c + 1], a.sl2, -ms));
              sum0 += p0;
              sum1 += p1;
              const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
              p[c / 2] = *reinterpret_cast<const uint32_t*>(&h);
            }
            tmem_st16(tS + c0 / 2, p);
          }
          l += sum0 + sum1;
          tmem_st_wait();
        }
        // values that some row does not see, and those behind the last entry that the last step reads
        const int v0 = max(low - t0, 0), v1 = min((end + 15) & ~15, KT);
        if (v0 < v1) {
          const int pl = pos + v_place(pair, j, f.n), st = pl % STAGES;
          wait(&full[st], pl / STAGES);
          __syncwarp();
          bool odd = false;
          for (int e = r; e < (v1 - v0) * VPR; e += SLOT) {
            const int row = v0 + e / VPR, c = e % VPR;
            uint4* at = reinterpret_cast<uint4*>(ring + st * TILE + (c >> 3) * PANEL + row * 128 +
                                                 ((c & 7) ^ (row & 7)) * 16);
            uint4 x = *at;
            if (odd_bf16x2(x.x) || odd_bf16x2(x.y) || odd_bf16x2(x.z) || odd_bf16x2(x.w)) {
              *at = make_uint4(without_odd(x.x), without_odd(x.y), without_odd(x.z), without_odd(x.w));
              odd |= row < end;
            }
          }
          if (__any_sync(FULL_MASK, odd) && lane == 0) odd_of[warp] = 1;
          fence_async_smem();
          // the slot's four warps: all of them have cleaned their share
          asm volatile("bar.sync %0, 128;" ::"r"(2 + s) : "memory");
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[s]);
      }
      if (tiles > 0) wait(&o_full[s], nO++);
      __syncwarp();
      tc_fence_after();
      float w0 = pair && s == 1 ? 0.f : 1.f, w1 = 1.f - w0;        // weights of the slots' sums
      if (!pair) {
        ml_of[s][r] = make_float2(m, l);
        tc_fence_before();
      }
      soft_sync();
      tc_fence_after();
      if (!pair) {
        const float2 x = ml_of[0][r], y = ml_of[1][r];
        m = fmaxf(x.x, y.x);
        const float ms = m == -INFINITY ? 0.f : m;
        w0 = ex2(x.x - ms);
        w1 = f.n > 1 ? ex2(y.x - ms) : 0.f;
        l = (x.x == m ? 1.f : w0) * x.y + (y.x == m ? 1.f : w1) * y.y;
      }
      int odd = 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) odd |= odd_of[w];

      const bool none = l == 0.f || (mine && row_idle(a, token));
      const float inv = none ? 0.f : 1.f / l;
      const long long at = f.slot * min(RT, f.prefix ? plan.R : plan.LG) + my;
      const long long row = (long long)token * (a.Hkv * a.G) + head;
      if (warp_live)
        for (int c = pair ? 0 : 32 * s; c < D; c += pair ? 32 : 64) {
          float o[32];
          if (pair) {
            tmem_ld32(tO + s * 128 + c, o);
          } else {
            tmem_ld32(tO + c, o);
            if (f.n > 1) {
              float y[32];
              tmem_ld32(tO + 128 + c, y);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = (w0 != 0.f ? w0 * o[i] : 0.f) + (w1 != 0.f ? w1 * y[i] : 0.f);
            }
          }
          if (mine) {
            if (odd && !f.prefix)
              for (int t = max(low, f.k0 * KT); t < min(lim, (f.k0 + f.n) * KT); ++t) {
                const __nv_bfloat16* vr = static_cast<const __nv_bfloat16*>(a.vo.p) + f.b * a.vo.seq +
                                          t * a.vo.tok + f.h * a.vo.head + c;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (c + i < D) {
                    const float x = __bfloat162float(vr[i]);
                    if (!isfinite(x)) o[i] += x;
                  }
              }
            if (f.whole) {
              __nv_bfloat16* to = static_cast<__nv_bfloat16*>(a.out) + row * D + c;
#pragma unroll
              for (int i = 0; i < 32; i += 8)
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
              float* to = (f.prefix ? a.part_p : a.part_o) + at * D + c;
#pragma unroll
              for (int i = 0; i < 32; i += 4)
                if (c + i < D) store4(to + i, make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]));
            }
          }
          __syncwarp();
        }
      if (mine && (pair || s == 0)) {
        if (f.whole) {
          if (a.lse) a.lse[row] = none ? -INFINITY : (m + log2f(l)) * (1.f / LOG2E);
        } else {
          (f.prefix ? a.ml_p : a.ml_o)[at] = make_float2(m, l);
        }
      }
      pos += 2 * f.n;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, TMEM_COLS);
  if (tid == 0)
    a.errs[blockIdx.x] = aborted ? BRISK_ERR_TIMEOUT : (bad && blockIdx.x == 0 ? BRISK_ERR_INVALID_ARG : BRISK_OK);
}

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

}  // namespace

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
