// Attention over a shared prefix and own caches, the attention weight that own entries got, and the
// eviction by it: arguments, the division of attention's work over the SMs, and the join of its parts.
#pragma once

#include <cuda.h>

#include "brisk_internal.cuh"

namespace brisk {

constexpr int CACHE_MAX_B = 4096;    // sequences of a call (the join's CTAs hold the tiles before each)
constexpr int CACHE_MAX_D = 128;     // width of a head
constexpr int CACHE_SMS = 152;
constexpr int UNIT_HEADS = 8;        // key heads of an own unit, at most

struct CacheView {   // element (s, t, h, :) at p + s*seq + t*tok + h*head, strides in elements
  const void* p;
  long long seq, tok, head;
};

// Division of 0 <= x < 2^31 by a constant of the call: floor(x / d) = (x * mul) >> (32 + shift) with
// mul = ceil(2^(32 + shift) / d) and 2^shift >= d, whose error is below x / 2^31 / d (Granlund and
// Montgomery, "Division by invariant integers using multiplication", PLDI'94). A dozen instructions fewer
// each than the compiler's division, in kernels that outgrow the instruction cache.
struct Divisor {
  unsigned long long mul;   // up to 2^33
  int d, shift;
  __host__ __device__ void set(int by) {
    d = by;
    shift = 0;
    while ((1LL << shift) < by) ++shift;
    mul = ((1ull << (32 + shift)) - 1) / by + 1;
  }
  __device__ __forceinline__ int of(int x) const {
    // mul = 2^32 + lo or less: x * mul in 64 bits
    const unsigned lo = (unsigned)mul, hi = (unsigned)(mul >> 32);
    const unsigned long long y = (unsigned long long)__umulhi((unsigned)x, lo) + (unsigned long long)(unsigned)x * hi;
    return (int)(y >> shift);
  }
};

// What the division of the work (see Plan) knows of a call before its lengths.
struct Shape {
  int kt, rt_p, rt_o;                // keys of a tile; rows of a tile over the prefix and over own caches
  int grid_p, grid_o;                // CTAs of the kernel for the prefix (0: the one for the own caches has both), of that
  int weight;
  int R, kP, nPT, nLT;               // rows a key head; key and row tiles of the prefix; row tiles of a sequence
  int log_kt, log_p, log_o;          // kt, rt_p and rt_o as powers of two (a weights call's rt_o is no power)
  int log_heads, slots_o;            // key heads of an own unit as a power of two; slots of each
  Divisor by_grid;                   // grid_o
  void set(int B, int LG, int P) {
    auto log2 = [](int x) { int l = 0; while ((2LL << l) <= x) ++l; return l; };
    R = B * LG;
    kP = (int)(((long long)P + kt - 1) / kt);
    nPT = P > 0 ? (int)(((long long)R + rt_p - 1) / rt_p) : 0;
    nLT = (int)(((long long)LG + rt_o - 1) / rt_o);
    log_kt = log2(kt);
    log_p = log2(rt_p);
    log_o = log2(rt_o);
    log_heads = slots_o = 0;
    by_grid.set(grid_o);
  }
};

struct AttendArgs {
  static constexpr bool PREFIX = true;   // units of a prefix's, and items filled up (see Plan)
  int B, L, G, Hkv, D, P, S;         // G query heads a key head
  int dt;                            // brisk_dtype of q, keys, values and out
  int joins;                         // the prefix's own kernel writes results (see JOIN_PARTS)
  Shape sh;
  CacheView q, kp, vp, ko, vo;
  Divisor by_L, by_G, by_LG;         // L, G and L * G
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
  int32_t* errs;                     // [grid_p + grid_o] what a CTA found wrong
  int32_t* status;
  long long wait_limit;
};

// ---------------------------------------------------------------- division of the work
// The unit of work is a tile of `kt` keys for a tile of up to `rt` query rows of one key head. A row is a
// (token, query head of the group) pair: row = token * G + g. Over the prefix, the rows of all
// sequences form common tiles (its keys are read once for rt_p rows, whichever sequence they are of);
// over the own caches, the rows of one sequence. The units stand in one sequence: first the prefix's
// (by head, row tile, key tile), then the own caches' (by sequence, head, row tile, key tile), and
// each CTA takes `share` of them, wherever that begins and ends; or the prefix's and the own caches' are two
// sequences of two kernels (apart), the own caches' first. A row tile's keys may so be divided over several CTAs,
// each of which leaves a part; the parts are joined by a merge kernel.
// Where there are CTAs to spare, attention's items (the keys of a row tile) are filled up to whole shares with units
// that hold nothing, so that no CTA has parts of two items, each with its own way from the first load to the stored
// part (a block of 32 positions over 4096 and 1100 entries 23.6 -> 19.5 us, 13 blocks of 7 over 3001 and up to 777 30.2
// -> 23.4). Where a prefix's unit takes far longer than an own one (fp32, few rows a sequence), it counts as `weight`
// units, in the CTA that has the first of them. (A share is at least a weight: no CTA between two of the prefix's
// parts is without one.)
// (An own unit may be the keys of several neighbouring heads at once, which a CTA's warps share: `own_heads` counts such
// groups then, and a slot is one for each of them, slots_o apart.)
// Slots: walking through a sequence, (item index + CTA) grows with every (item, CTA) pair, so it
// numbers the parts. Counts of units fit 31 bits (checked on the host).
struct Plan {
  int B, LG, Hkv;
  int nPT, kP, nLT, R;               // as Shape's
  int kPp;                           // units of a row tile over the prefix: kP, filled up
  int UP, UO;                        // units of the prefix and of the own caches
  int own0;                          // number of the own caches' first unit
  int weight;                        // units that one of the prefix's counts as
  int share_p, share_o;              // units a CTA
  int own_heads;                     // key heads of the own caches, or groups of them
  int filled;                        // what items are filled up to a multiple of
  bool apart;                        // the prefix's units and the own caches' are two sequences

  Plan() = default;
  // (own_tiles: of all sequences, filled up to multiples of pad)
  template <typename Args>
  __device__ Plan(const Args& a, int own_tiles, int pad) {
    const Shape& sh = a.sh;
    B = a.B; LG = a.L * a.G; Hkv = a.Hkv; nLT = sh.nLT; R = sh.R;
    nPT = Args::PREFIX ? sh.nPT : 0;
    kP = Args::PREFIX ? sh.kP : 0;
    apart = Args::PREFIX && sh.grid_p > 0;
    filled = Args::PREFIX ? pad : 1;
    kPp = apart ? kP : fill(kP, pad);
    own_heads = Args::PREFIX ? Hkv >> sh.log_heads : Hkv;
    UP = Hkv * nPT * kPp;
    UO = own_heads * nLT * own_tiles;
    weight = 1;
    if (Args::PREFIX && pad == 1 && sh.weight > 1) {
      // an own fragment costs about one and a half of its units more, whatever its length (rounded alike in all kernels)
      const float t = (float)own_tiles;
      const int w = max(1, (int)__fdiv_rn(__fmul_rn(t, (float)sh.weight), __fadd_rn(t, __fmul_rn(1.5f, (float)B))));
      const unsigned all = (unsigned)UP * w + UO;            // (UP and UO: up to 2e9 together)
      if (UP < (1 << 28) && all < 0x7ffff000u && sh.by_grid.of(all) >= w) weight = w;
    }
    own0 = apart ? 0 : UP * weight;
    share_o = max(1, sh.by_grid.of(own0 + UO + sh.grid_o - 1));
    share_p = apart ? max(1, (UP + sh.grid_p - 1) / sh.grid_p) : share_o;
  }
  __device__ static int fill(int n, int pad) { return pad == 1 ? n : (n + pad - 1) / pad * pad; }
  // Of a plan whose items are not filled up: its share, if filling them up to a multiple of it lets no CTA's share
  // grow; else 1.
  __device__ int fill_to(int grid_o) const {
    if (share_o == 1) return 1;
    const long long items = (long long)own_heads * nLT * B + (apart ? 0 : (long long)Hkv * nPT);
    return weight == 1 && (long long)own0 + UO + items * (share_o - 1) <= (long long)share_o * grid_o ? share_o : 1;
  }
};

// The units a CTA has of a sequence of `all`.
__device__ __forceinline__ int2 units_of(int cta, int share, int all) {
  const long long first = (long long)cta * share;
  return make_int2((int)min(first, (long long)all), (int)min(first + share, (long long)all));
}

// A CTA's share of one item (a row tile's keys): key tiles [k0, k0 + n).
struct Frag {
  int prefix, whole, last;           // whole: no other part for these rows exists; last: of the CTA
  int h, b, k0, n;
  int row0, rows;                    // rows of the head over the prefix, of the sequence else
  int slot, len;                     // len: entries of the prefix, or in use of the own cache
};

// The sequence of a CTA's first own unit, and the key tiles of the sequences before it (see make_plan).
struct Start { int b, before; };

template <typename Args>
__device__ __forceinline__ int clamped_len(const Args& a, int b) {
  return min(max(a.own_len[b], 0), a.S);
}
template <typename Args>
__device__ __forceinline__ int tiles_of(const Args& a, int len) {
  return (len + a.sh.kt - 1) >> a.sh.log_kt;
}

// Walks through a CTA's units: the prefix's (unless another kernel has them, apart), then the own caches'.
struct Walk {
  int pu, pend;                      // the prefix's next unit and their end
  int u, end, c, b, base, n, len;    // the own ones'; b: sequence whose units begin at `base`, n for a row tile
  int later;                         // the next sequence's length, on its way

  Walk() = default;
  template <typename Args>
  __device__ Walk(const Args& a, const Plan& p, int cta, const Start& start) {
    const int2 r = units_of(cta, p.share_o, p.own0 + p.UO);
    pu = pend = 0;
    if (Args::PREFIX && !p.apart && r.x < p.own0) {
      pu = (r.x + p.weight - 1) / p.weight;
      pend = (min(r.y, p.own0) + p.weight - 1) / p.weight;
    }
    u = max(r.x, p.own0);
    end = r.y;
    c = cta;
    b = base = n = len = later = 0;
    if (u < end) {                   // (a CTA without own units has no start)
      b = start.b;
      base = p.own0 + p.own_heads * p.nLT * start.before;
      len = clamped_len(a, b);
      n = Plan::fill(tiles_of(a, len), p.filled);
      later = a.own_len[min(b + 1, a.B - 1)];
    }
  }
  template <typename Args>
  __device__ bool next(const Args& a, const Plan& p, Frag& f) {
    if constexpr (Args::PREFIX) if (pu < pend) {
      const int item = pu / p.kPp, stop = min((item + 1) * p.kPp, pend);
      f.prefix = 1;
      f.k0 = pu - item * p.kPp;
      f.n = min(p.kP - f.k0, stop - pu);
      f.h = item / p.nPT;
      f.b = 0;
      f.row0 = (item - f.h * p.nPT) * a.sh.rt_p;
      f.rows = min(a.sh.rt_p, p.R - f.row0);
      f.slot = item + c;
      f.whole = f.n == p.kP && a.S == 0;
      f.len = a.P;
      pu = stop;
      f.last = pu >= pend && u >= end;
      return true;
    }
    if (u >= end) return false;
    const int per = p.own_heads * p.nLT;
    while (u >= base + per * n) {
      base += per * n;
      ++b;
      len = min(max(later, 0), a.S);
      n = Plan::fill(tiles_of(a, len), p.filled);
      later = a.own_len[min(b + 1, a.B - 1)];
    }
    const int r = (u - base) / n, tile = r % p.nLT, real = tiles_of(a, len), stop = min(base + (r + 1) * n, end);
    f.prefix = 0;
    f.b = b;
    f.h = r / p.nLT;
    f.k0 = u - base - r * n;
    f.n = min(real - f.k0, stop - u);
    f.row0 = tile * a.sh.rt_o;
    f.rows = min(a.sh.rt_o, p.LG - f.row0);
    f.slot = b * per + r + c;
    f.whole = f.n == real && p.UP == 0;
    f.len = len;
    u = stop;
    f.last = u >= end;
    return true;
  }
};

// A part's sums lie by groups of four columns, then rows: [D / 4][rows of a slot][4], so that neighbouring
// rows, which are neighbouring lanes of the kernels on both sides, lie side by side.
__device__ __forceinline__ long long part_at(long long slot, int per, int D, int row, int c) {
  return slot * per * D + ((long long)(c >> 2) * per + row) * 4;
}

// Token (b * L + i) and query head of a fragment's row, and how many keys the row sees.
__device__ __forceinline__ void row_of(const AttendArgs& a, const Frag& f, int r, int& token, int& head) {
  const int row = f.row0 + r, t = a.by_G.of(row);
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

// The plan of a call, by all THREADS threads of a CTA: sums the sequences' key tiles and finds the sequence of the first
// own unit of `cta` (-1: not asked for) in shared memory, valid after the call. The tiles before each sequence go to
// `cum` unless that is nullptr; *bad is set where a length lies outside 0..S (the caller clears it before a barrier).
template <int THREADS, typename Args>
__device__ Plan make_plan(const Args& a, int cta, int32_t* cum, int* warp_sum, int* bad, Start* start) {
  const int per = (a.B + THREADS - 1) / THREADS, tid = threadIdx.x, lane = tid & 31;
  const int b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
  const int mine = b0 < b1 ? a.own_len[b0] : 0;    // (seldom more than one a thread)
  auto tiles = [&](int b, int pad) {
    const int len = b == b0 ? mine : a.own_len[b];
    if (len < 0 || len > a.S) *bad = 1;
    return Plan::fill(tiles_of(a, min(max(len, 0), a.S)), pad);
  };
  int pad = 1, before, total;
  Plan plan;
  for (;;) {
    int sum = 0;
    for (int b = b0; b < b1; ++b) sum += tiles(b, pad);
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(FULL_MASK, run, o);
      if (lane >= o) run += x;
    }
    if (lane == 31) warp_sum[tid >> 5] = run;
    __syncthreads();
    before = run - sum;
    total = 0;
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < (tid >> 5)) before += warp_sum[w];
      total += warp_sum[w];
    }
    plan = Plan(a, total, pad);
    if (pad > 1) break;
    if constexpr (Args::PREFIX) pad = plan.fill_to(a.sh.grid_o);
    if (pad == 1) break;
    __syncthreads();                               // the sums are read
  }
  const int at = cta < 0 ? -1 : max(0, units_of(cta, plan.share_o, plan.own0 + plan.UO).x - plan.own0) / (plan.own_heads * plan.nLT);
  for (int b = b0; b < b1; ++b) {
    const int n = tiles(b, pad);
    if (cum) cum[b] = before;
    if (at >= before && at < before + n) *start = Start{b, before};
    before += n;
  }
  if (cum && tid == 0) cum[a.B] = total;
  __syncthreads();
  return plan;
}

// Parts of a row's own entries that the prefix's kernel joins itself, where it has all the prefix for the row;
// with more, whose loads would wait for one another, it leaves a part too (128 blocks of 32 positions over 8192 + 256
// to 1024 entries: none 459 us, one or two 440).
constexpr int JOIN_PARTS = 2;

// The parts of row `r` of a head, over the prefix or over the own entries: a run of `n` slots.
struct Parts {
  int n, per;
  const float* sums;                 // column 0 of the first part; the next one is per * D further
  const float2* ml;
};
// (by_share_p, by_share_o: the plan's)
__device__ __forceinline__ Parts prefix_parts(const AttendArgs& a, const Plan& p, const Divisor& by_share_p, int h, int r) {
  Parts x{0, min(a.sh.rt_p, p.R), nullptr, nullptr};
  if (p.kP == 0) return x;
  const int pt = r >> a.sh.log_p, first = (h * p.nPT + pt) * p.kPp;
  const int c0 = by_share_p.of(first * p.weight), slot = h * p.nPT + pt + c0;
  x.n = by_share_p.of((first + p.kPp - 1) * p.weight) - c0 + 1;
  x.sums = a.part_p + part_at(slot, x.per, a.D, r - (pt << a.sh.log_p), 0);
  x.ml = a.ml_p + (long long)slot * x.per + (r - (pt << a.sh.log_p));
  return x;
}
// (cum as make_plan leaves it)
__device__ __forceinline__ Parts own_parts(const AttendArgs& a, const Plan& p, const Divisor& by_share_o, const int32_t* cum,
                                           int h, int r) {
  Parts x{0, min(a.sh.rt_o, p.LG), nullptr, nullptr};
  const int b = a.by_LG.of(r), before = cum[b], n = cum[b + 1] - before;
  if (n == 0) return x;
  const int group = h >> a.sh.log_heads;
  const int ro = r - b * p.LG, lt = ro >> a.sh.log_o, of = group * p.nLT + lt, per = p.own_heads * p.nLT;
  const int u = p.own0 + per * before + of * n, c0 = by_share_o.of(u);
  const int slot = b * per + of + c0 + (h - (group << a.sh.log_heads)) * a.sh.slots_o;
  x.n = by_share_o.of(u + n - 1) - c0 + 1;
  x.sums = a.part_o + part_at(slot, x.per, a.D, ro - (lt << a.sh.log_o), 0);
  x.ml = a.ml_o + (long long)slot * x.per + (ro - (lt << a.sh.log_o));
  return x;
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

// Keys of a tile, rows of it, and CTAs: bf16 on the tensor cores, fp32 on the FMA units. With bf16 and more
// than SLOT_ROWS query rows a key head, the prefix has a kernel of its own from apart_units() of its units on.
// That kernel reads a key tile for twice the rows, but is one more launch, divides the prefix by itself, in whole
// rounds of CTAs, and leaves rows with more than JOIN_PARTS own parts to the join. 32 query heads on 8, own caches with
// room S, half of it to all in use, R rows a key head; U units of it take, with and without it, us:
//   S 60 (0 to 60; 32 rows a sequence): R 512, U 512: 29.6 and 29.8; 768: 32.1, 38.8; 1024: 38.6, 47.6; 2048: 49.8, 76.5;
//     R 2048: 512: 35.3, 38.2; 1024: 44.2, 55.7; 2048: 53.8, 84.6
//   S 500, R 1024, 32 rows: U 512: 36.4, 32.7; 1024: 47.0, 42.0; 2048: 58.4, 64.2; 4096: 78.5, 97.7;
//     R 4096, 128 rows: 512: 44.9, 47.1; 2048: 70.6, 82.7
//   S 640, R 1024, 32 rows: U 1024: 49.4, 44.5; 2048: 59.1, 60.4; 4 rows: 1024: 125.6, 117.0; 2048: 134.9, 130.6
//   S 800, R 1024, 32 rows: U 1024: 53.4, 44.2; 2048: 62.6, 58.1; 4096: 83.3, 88.2
//   S 2048, R 1024, 32 rows: U 512: 62.9, 50.7; 1024: 72.7, 57.0; 2048: 81.8, 70.7; 4096: 101, 102; 8192: 150, 154;
//     128 rows: 1024: 49.6, 37.1; 4096: 79.9, 82.4; 4 rows: 512: 277, 278; 4096: 314, 340.
// Between the borders either side may be ahead by a tenth, as the rounds come out.
constexpr int TC_KT = 128, SLOT_ROWS = 128, PAIR_ROWS = 256, SIMT_KT = 64, SIMT_ROWS = 64;
constexpr int SLOT_CTAS = 2 * CACHE_SMS;             // (the fp32 kernel's, too)
constexpr int APART_UNITS = 3 * CACHE_SMS;           // own caches whose parts it joins whatever their division
constexpr int APART_UNITS_SOME = 8 * CACHE_SMS;      // up to SOME_TILES of own keys
constexpr int APART_UNITS_LONG = 24 * CACHE_SMS;
constexpr int SOME_TILES = 5;
inline int apart_units(int S) {
  return S <= JOIN_PARTS * TC_KT ? APART_UNITS : (S <= SOME_TILES * TC_KT ? APART_UNITS_SOME : APART_UNITS_LONG);
}
// fp32: up to FEW_ROWS rows of a sequence have a form of their own (64 single tokens, 32 heads on 8, D = 128, over
// 1000 to 2000 own and 2000 shared entries: 216 us, with the form for more rows 685 us). One of its units takes about
// a sixth (up to 4 rows) or a fourth of the time of a prefix's unit of a full tile, where own caches are long: counting
// the latter as 1, 4, 5 and 6 units 571, 239, 215 and 216 us, 8 rows 626, 366, 399 and 429 us.
constexpr int FEW_ROWS = 8;
inline void divide(AttendArgs* a) {
  const bool tc = a->dt == BRISK_DT_BF16;
  const long long R = (long long)a->B * a->L * a->G;
  const long long units = a->Hkv * ((R + PAIR_ROWS - 1) / PAIR_ROWS) * (((long long)a->P + TC_KT - 1) / TC_KT);
  const bool apart = tc && R > SLOT_ROWS && units >= apart_units(a->S);
  const int rows = a->L * a->G;
  a->sh.kt = tc ? TC_KT : SIMT_KT;
  a->sh.rt_o = tc ? SLOT_ROWS : SIMT_ROWS;
  a->sh.rt_p = apart ? PAIR_ROWS : a->sh.rt_o;
  a->sh.grid_p = apart ? CACHE_SMS : 0;
  a->joins = 1;
  a->sh.grid_o = SLOT_CTAS;
  a->sh.weight = !tc && R > FEW_ROWS && rows <= FEW_ROWS ? (rows <= 4 ? 6 : 4) : 1;
  a->sh.set(a->B, rows, a->P);
}

// A tile of 128 rows in shared memory, as the products read it: panels of 64 columns, 128 bytes a row, the
// 16-byte pieces of which are swizzled.
constexpr int TILE_PANEL = 128 * 128;
// A warp's 32 queries (a row a lane, from nullptr: none) on their way to rows row0.. of a tile: 4 lanes a row, 64
// bytes of it at a time. Columns up to a multiple of 16, which the products read, are zeros.
template <int DP>
__device__ __forceinline__ void fetch_queries(const __nv_bfloat16* q, int D, uint8_t* tile, int row0) {
  const int lane = threadIdx.x & 31, np = 2 * ((D + 15) / 16);       // 16-byte pieces that the products read
#pragma unroll 1
  for (int i = 0; i < 32; i += 8) {
    const int in = i + (lane >> 2), at = row0 + in;
    const unsigned long long from = __shfl_sync(FULL_MASK, reinterpret_cast<unsigned long long>(q), in);
    if (from)
#pragma unroll
      for (int k = 0; k < DP / 32; ++k) {
        const int c = 4 * k + (lane & 3);
        const uint32_t to = su32(tile + at * 128 + (c >> 3) * TILE_PANEL + ((c ^ at) & 7) * 16);
        if (8 * c < D)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from + 16 * c) : "memory");
        else if (c < np)
          asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0) : "memory");
      }
  }
}

// 16 bytes on their way to shared memory, past L1; zeros where there is nothing to copy (`from` is valid anyway).
__device__ __forceinline__ void copy16(float* to, const float* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(su32(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}
// A tile of fp32 keys or values, by all threads of a CTA; zeros behind the last entry.
template <int ROWS, int THREADS>
__device__ __forceinline__ void copy_tile(float* to, int stride, const float* from, long long tok, int t0, int len, int nv) {
#pragma unroll 4
  for (int e = threadIdx.x; e < ROWS * nv; e += THREADS) {
    const int r = e / nv, c = 4 * (e - r * nv);
    const bool there = t0 + r < len;
    copy16(to + r * stride + c, there ? from + (t0 + r) * tok + c : from, there);
  }
}

// Tensor map of a cache's tiles of 64 columns x 128 entries (cache_attend_tc.cu).
bool make_cache_map(CUtensorMap* map, const CacheView& v, int D, int heads, int toks, int seqs);

// The next kernel of the stream may be set up once all of this one's CTAs have begun; the wait until
// the kernel before has ended, and what it wrote can be read.
__device__ __forceinline__ void let_next_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Launches a kernel that may be set up while the one before it on the stream still runs.
template <typename Kernel, typename... Args>
inline cudaError_t launch_early(Kernel kernel, dim3 grid, int threads, size_t smem, cudaStream_t stream, bool early,
                                const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t stream);
cudaError_t launch_attend_f32(const AttendArgs& a, cudaStream_t stream);
// The prefix alone (sh.grid_p CTAs), behind the kernel that has the own caches' units.
cudaError_t launch_prefix_tc(const AttendArgs& a, cudaStream_t stream);
cudaError_t launch_prefix_f32(const AttendArgs& a, cudaStream_t stream);
cudaError_t launch_merge(const AttendArgs& a, cudaStream_t stream);

// ---------------------------------------------------------------- attention weight of own entries
struct WeightArgs {
  static constexpr bool PREFIX = false;  // (128 sequences of 1024 to 4096 entries: 132 us, items filled up 138)
  int B, L, G, Hkv, D, S, dt;
  Shape sh;
  CacheView q, ko;
  Divisor by_G;
  const int32_t *own_len, *visible;
  const float* lse;        // [B, L, Hkv * G]
  float scale, sl2, decay;           // sl2: scale * log2(e)
  const float* acc_in;     // [B, Hkv, S] or nullptr (zeros)
  float* acc_out;          // [B, Hkv, S]
  int32_t* status;
  long long wait_limit;
};
inline void divide(WeightArgs* a) {
  const int rows = a->L * a->G;
  a->sh.kt = TC_KT;
  a->sh.rt_p = a->sh.weight = 1;
  a->sh.rt_o = rows;                 // all rows of a sequence are one tile
  a->sh.grid_p = 0;
  a->sh.grid_o = CACHE_SMS;
  a->sh.set(a->B, rows, 0);
}
cudaError_t launch_weights_tc(const WeightArgs& a, cudaStream_t stream);
cudaError_t launch_weights_f32(const WeightArgs& a, cudaStream_t stream);

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
