// Attention over own caches in 4 bits, for the rows of a few queries: parts (or results) of up to 8 rows of a key head
// against the keys of a fragment (see Plan), as the kernels of unquantised caches leave them.
//
// Eight warps of a CTA share the heads of a unit (see divide_packed); the warps of a head take 32 of its keys each in
// turn. The codes become fp16 in registers, in the places where mma.sync wants them, and never pass through shared memory
// as numbers: at the rate at which memory delivers codes, a tile of fp16 written and read there would take more than the
// bandwidth it has. (tcgen05 takes its tiles of keys from shared memory alone, and 128 rows of queries where there are
// 1 to 16.) The products are
//   S^T [16 keys, 8 rows]      = K [16 keys, D] Q^T,
//   O^T [D channels, 8 rows]  += V^T [D channels, 16 keys] P^T.
// The order of k in a product is free, so a lane of K has 32 neighbouring channels of its key, 16 bytes of codes, and a
// lane of V 16 neighbouring channels of four keys, whose codes are paired by key before they are converted.
//
// K and V are exact in fp16. A row of Q is scaled by a power of two to a magnitude of 2^14 to 2^15, where steps of fp16 end at
// 2^-24: bf16 is exact then from 2^-31 of the row's largest on, and fp32 (TERMS = 2) goes as a sum of two fp16 of 11 bits
// each, off by 2^-23 of itself; what is smaller by up to 2^-25, 2^-39 of the largest. Weights are taken relative to
// 2^-SHIFT of the held maximum; rounding them costs 2^-11 each (fp32: two terms, less than 2^-22), or that 2^-25, which is
// 2^-35 of the maximum, if it is more. Sums, maxima and S are fp32. With fp32 every 16 keys' sums are taken anew and added in
// fp32, since the tensor cores cut what they add to a sum towards zero.
//
// Keys and values come through a ring of a warp's own, in which its lanes copy 16 bytes at a time, a place of 32 keys
// ahead, across the ends of fragments: nobody waits for another but where the parts of a head's warps meet.
// Entries that a row does not see: scores are masked by selection, and the scales of the values of a step of which some
// row does not see all are cut to ones that stand for numbers, so that what is left in the ring or the cache cannot
// defeat a weight of 0.
//
// Bound by the instructions of a step and their latencies with four warps a scheduler, not by bytes (which are few):
// 256 instructions for 16 keys of a head of 128, of which 93 wait their turn for the units of integer logic (the
// conversions take these two cycles each) and 16 are products; 474 cycles, 357 without the copies. Single tokens of 256
// sequences over 512 to 2048 own and 2048 shared entries take 104 us, 377 MB of codes among it (0.6 us less without the
// factors that leave out channels that are not there); one over 130001 entries 43 us, 3.5 TB/s. Steps of 16 keys with
// three CTAs an SM (125 and 54 us) and a third place in the ring (106 and 45) did not help.
#include "packed.cuh"

namespace brisk {
namespace {

constexpr int WARPS = PACKED_WARPS, THREADS = 32 * WARPS;
constexpr int STEP = 32, HALVES = STEP / 16;        // keys that a warp takes at a time
constexpr int STAGES = 2;
constexpr int AHEAD = 4;                           // fragments that a warp's copies may be ahead, a power of two
constexpr float LAZY = 5.f, SHIFT = 10.f;          // log2 of what a score may exceed the held maximum by; weights below 2^15

// A form of the kernel. DP: 64 or 128 channels, of which a row's first D are there. TERMS: fp16 numbers that make up a query
// and a weight. QUAD: up to four rows, each of which has two columns of the products.
template <int DP_, int TERMS_, bool QUAD_>
struct Form {
  static constexpr int DP = DP_, TERMS = TERMS_, QUAD = QUAD_;
  static constexpr int ROWS = QUAD ? 4 : 8;
  static constexpr int ROW = DP / 2, SROW = DP / 16;
  static constexpr int CODES = STEP * ROW, SCALES = STEP * SROW;
  static constexpr int VALUES = CODES + SCALES;    // of a tile: where the values' begin
  static constexpr int BYTES = 2 * VALUES;
};
constexpr int OS = CACHE_MAX_D + 4;                // floats between rows of a warp's sums
template <typename T>
struct Smem {
  alignas(16) uint8_t ring[WARPS][STAGES * T::BYTES];
  float sums[WARPS][T::ROWS][OS];
  float2 ml[WARPS][T::ROWS];
  Walk walk[WARPS];
  Frag frag[WARPS][AHEAD];
};

// Key of a product's row i (of 8): lanes g = 2j and 2j + 1 of K, and the lanes c of V with their first and their second
// keys, so read shared memory without conflicts.
__device__ __forceinline__ int key_of(int i) { return (0x53427160 >> (4 * i)) & 7; }
// A 16-byte piece's place in a tile of codes: with 64 bytes a row, pieces of 128-byte lines are swapped.
template <int DP>
__device__ __forceinline__ int piece_at(int key, int piece) {
  if (DP == 64) return key * 32 + piece * 16;
  return (key >> 1) * 128 + ((((key & 1) << 2 | piece) ^ (2 * ((key >> 1) & 3))) << 4);
}

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {   // to a sum of 0
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {   // of an 8 x 8 matrix of 16 bits
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 floats_of(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }

template <int N>
__device__ __forceinline__ void copy_bytes(void* to, const void* from) {
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(su32(to)), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(su32(to)), "l"(from), "n"(N) : "memory");
}

// A lane's share of copying the codes and scales of STEP keys and values to a place of the ring: where from, of those that
// are next. Rows from the cache's end on are left as they are.
template <typename T>
struct Copies {
  static constexpr int DP = T::DP, VALUES = T::VALUES;
  static constexpr int P = DP / 32;                // 16-byte pieces a row
  const uint8_t *k, *v, *ks, *vs;
  int left;                                        // keys of the fragment from the first of these on
  // (one multiplication of 32 bits each, beside the conversions that take the integer units)
  static __device__ __forceinline__ const uint8_t* ahead(const uint8_t* p, int rows, uint32_t stride) {
    return p + (unsigned long long)(uint32_t)rows * stride;
  }
  __device__ __forceinline__ void begin(const PackedArgs& p, const Frag& f, int t0, int end) {
    const int lane = threadIdx.x & 31;
    const bool wide = (p.a.D & 31) == 0;           // (else rows start on 8 bytes)
    const int row = t0 + (wide ? lane / P : lane / (2 * P)), at = wide ? 16 * (lane % P) : 8 * (lane % (2 * P));
    k = ahead(p.k.codes + f.b * p.k.seq + f.h * p.k.head + at, row, p.k.tok);
    v = ahead(p.v.codes + f.b * p.v.seq + f.h * p.v.head + at, row, p.v.tok);
    ks = ahead(p.k.scales + f.b * p.k.sseq + f.h * p.k.shead, t0 + lane, p.k.stok);
    vs = ahead(p.v.scales + f.b * p.v.sseq + f.h * p.v.shead, t0 + lane, p.v.stok);
    left = end - t0;
  }
  __device__ __forceinline__ void copy_scales(uint8_t* to) const {
    const int at = T::CODES + (threadIdx.x & 31) * T::SROW;
    copy_bytes<T::SROW>(to + at, ks);
    copy_bytes<T::SROW>(to + VALUES + at, vs);
  }
  __device__ __forceinline__ void copy(const PackedArgs& p, uint8_t* to, int step) {
    const int lane = threadIdx.x & 31;
    if (p.a.D == DP && left >= STEP) {             // nothing to leave out
      uint8_t* at = to + piece_at<DP>(lane / P, lane % P);
      constexpr int R = 32 / P;                    // rows at once; the next are 512 bytes further
#pragma unroll
      for (int i = 0; i < STEP / R; ++i) {
        copy_bytes<16>(at + 512 * i, ahead(k, R * i, p.k.tok));
        copy_bytes<16>(at + 512 * i + VALUES, ahead(v, R * i, p.v.tok));
      }
      copy_scales(to);
    } else {
      const bool wide = (p.a.D & 31) == 0;
      const int n = wide ? P : 2 * P, row = lane / n, piece = lane % n, bytes = wide ? 16 : 8;
#pragma unroll 1
      for (int r = row; r < STEP; r += 32 / n)
        if (r < left && bytes * piece < p.a.D / 2) {
          uint8_t* at = wide ? to + piece_at<DP>(r, piece) : to + piece_at<DP>(r, piece >> 1) + 8 * (piece & 1);
          const uint8_t *kf = ahead(k, r - row, p.k.tok), *vf = ahead(v, r - row, p.v.tok);
          if (wide) {
            copy_bytes<16>(at, kf);
            copy_bytes<16>(at + VALUES, vf);
          } else {
            copy_bytes<8>(at, kf);
            copy_bytes<8>(at + VALUES, vf);
          }
        }
      if (lane < left) copy_scales(to);
    }
    k = ahead(k, step, p.k.tok);
    v = ahead(v, step, p.v.tok);
    ks = ahead(ks, step, p.k.stok);
    vs = ahead(vs, step, p.v.stok);
    left -= step;
  }
};

template <typename T>
__global__ void __launch_bounds__(THREADS, 2)
packed_few_kernel(const __grid_constant__ PackedArgs p) {
  constexpr int DP = T::DP, TERMS = T::TERMS, ROWS = T::ROWS;
  constexpr bool QUAD = T::QUAD;
  constexpr int KS = DP / 16;                      // steps of 16 channels of a score
  constexpr int OT = QUAD ? DP / 32 : KS;          // tiles of O
  constexpr int R = QUAD ? 1 : 2;                  // rows of a lane
  const AttendArgs& a = p.a;
  extern __shared__ __align__(16) uint8_t raw[];
  Smem<T>& sm = *reinterpret_cast<Smem<T>*>(raw);
  __shared__ int warp_sum[WARPS], bad;
  __shared__ Start start;
  __shared__ Plan plan;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3, D = a.D;
  if (tid == 0) bad = 0;
  __syncthreads();
  let_next_begin();
  {
    const Plan made = make_plan<THREADS>(a, blockIdx.x, blockIdx.x == 0 ? a.cum : nullptr, warp_sum, &bad, &start);
    if (tid == 0) plan = made;
  }
  __syncthreads();
  if (tid == 0) a.errs[a.sh.grid_p + blockIdx.x] = bad && blockIdx.x == 0 ? BRISK_ERR_INVALID_ARG : BRISK_OK;

  Walk& walk = sm.walk[warp];
  Frag* frags = sm.frag[warp];
  if (lane == 0) walk = Walk(a, plan, blockIdx.x, start);
  int walked = 0, done = 0;                        // fragments found, and worked through
  bool more = true;                                // there may be another one to find
  auto find = [&]() {                              // the next fragment, into its place (there is room)
    int ok = 0;
    if (lane == 0) ok = walk.next(a, plan, frags[walked % AHEAD]);
    more = __shfl_sync(FULL_MASK, ok, 0) != 0;     // (and the lanes see it)
    __syncwarp();
    walked += more;
    return more;
  };

  // the copying side: fragment number cf, what is left of it for this warp, the place that is filled next
  const int heads = 1 << a.sh.log_heads, sub = warp & (heads - 1), group = WARPS >> a.sh.log_heads, turn = warp >> a.sh.log_heads;
  const int stride = STEP * group;                 // keys of the warps of a head: each has every group-th STEP
  int cf = -1;
  Copies<T> next;
  next.left = 0;
  int pending = 0;                                 // tiles of the ring that are not read yet
  uint8_t* const ring = sm.ring[warp];
  int write = 0, read = 0;                         // places of the next one copied, and of the next one read
  auto issue = [&]() {                             // one more tile, as a group of copies; false: there is none (yet)
    while (next.left <= 0) {
      if (cf + 1 == walked && (!more || walked - done >= AHEAD || !find())) return false;
      ++cf;
      Frag f = frags[cf % AHEAD];
      f.h = f.h * heads + sub;
      next.begin(p, f, (f.k0 << a.sh.log_kt) + turn * STEP, min(f.len, (f.k0 + f.n) << a.sh.log_kt));
    }
    next.copy(p, ring + write, stride);
    asm volatile("cp.async.commit_group;" ::: "memory");
    write ^= T::BYTES;
    ++pending;
    return true;
  };
  auto meet = [&]() {                              // of the warps of a head
    if (group == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + sub), "r"(32 * group) : "memory");
  };
  static_assert(STAGES == 2, "places alternate");

  // where a lane reads a tile: its key's codes and scales, and those of its two values (each 8 and 16 rows further, too)
  constexpr int VALUES = T::VALUES;
  int at_k = DP == 128 ? piece_at<DP>(key_of(g), c) : key_of(g) * T::ROW + 8 * c, at_ks = T::CODES + key_of(g) * T::SROW + c * (DP / 64);
  int at_v[2], at_vs[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int key = key_of(2 * c + i);
    at_v[i] = VALUES + (DP == 128 ? piece_at<DP>(key, g >> 1) + 8 * (g & 1) : key * T::ROW + 4 * g);
    at_vs[i] = VALUES + T::CODES + key * T::SROW + g * (DP / 8) / GROUP;
  }
  // of two weights of a row, the first and the second in the half that the lane's column stands for
  const uint32_t pick[2] = {g & 1 ? 0x1044u : 0x4410u, g & 1 ? 0x3244u : 0x4432u};
  // (the compiler would rather work them out again at every step)
  asm volatile("" : "+r"(at_k), "+r"(at_ks), "+r"(at_v[0]), "+r"(at_v[1]), "+r"(at_vs[0]), "+r"(at_vs[1]));
  // What a byte of a key's scales is multiplied by (see scale_plain): 0 from channel D on, where the byte is not in use and
  // may be anything, so that the queries' zeros meet zeros. (Codes of what is not there are numbers, whatever they are.)
  uint32_t there[DP / 64];
#pragma unroll
  for (int j = 0; j < DP / 64; ++j) there[j] = c * (DP / 4) + GROUP * j < D ? SCALE_PLAIN : 0;

  for (;;) {
    if (walked == done && (!more || !find())) break;
#pragma unroll 1
    while (pending < STAGES && issue()) {}
    Frag f = frags[done % AHEAD];
    f.h = f.h * heads + sub;
    const int end = min(f.len, (f.k0 + f.n) << a.sh.log_kt);

    // queries: lane (g, c) has channels (DP / 4) c .. of row g (QUAD: g / 2); row_scale: of rows 2c, 2c + 1 (c)
    const int qrow = QUAD ? g >> 1 : g;
    uint32_t qf[TERMS][KS][2];
    float row_scale[R];
    int see = f.len, low;                          // entries that row qrow sees, and the row that sees fewest
    {
      float q[DP / 4];
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < DP / 4; ++i) q[i] = 0.f;
      if (qrow < f.rows) {
        int token, head;
        row_of(a, f, qrow, token, head);
        see = row_limit(a, f, token, f.len);
        const int b = a.by_L.of(token), i = token - b * a.L;
        const long long at = b * a.q.seq + i * a.q.tok + head * a.q.head + c * (DP / 4);
#pragma unroll
        for (int i = 0; i < DP / 4; i += 4)
          if (c * (DP / 4) + i < D) {
            const float4 x = TERMS == 1 ? load4(static_cast<const __nv_bfloat16*>(a.q.p) + at + i)
                                        : load4(static_cast<const float*>(a.q.p) + at + i);
            q[i] = x.x; q[i + 1] = x.y; q[i + 2] = x.z; q[i + 3] = x.w;
          }
#pragma unroll
        for (int i = 0; i < DP / 4; ++i) top = __uint_as_float(max(__float_as_uint(top), __float_as_uint(q[i]) & 0x7fffffffu));
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1)
        top = __uint_as_float(max(__float_as_uint(top), __shfl_xor_sync(FULL_MASK, __float_as_uint(top), o)));
      const int up = query_shift(__float_as_uint(top));
      const float by = exp2_of(up), mine = query_scale(a.sl2, up);
#pragma unroll
      for (int i = 0; i < DP / 4; i += 2) {
        const float x = q[i] * by, y = q[i + 1] * by;
        const uint32_t h = half2_of(x, y);
        qf[0][i / 4][(i >> 1) & 1] = h;
        if constexpr (TERMS == 2) {
          const float2 z = floats_of(h);
          qf[TERMS - 1][i / 4][(i >> 1) & 1] = half2_of(x - z.x, y - z.y);
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) row_scale[r] = __shfl_sync(FULL_MASK, mine, 4 * (2 * c + r));
      low = __reduce_min_sync(FULL_MASK, see);
    }

    float l[R], above[R], less[R];                 // (above: what a score is compared with, less: what is added to it)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      l[r] = less[r] = 0.f;
      above[r] = -INFINITY;
    }
    float o[OT][4];
#pragma unroll
    for (int i = 0; i < OT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.f;

    for (int t0 = (f.k0 << a.sh.log_kt) + turn * STEP; t0 < end; t0 += stride) {
      __syncwarp();                                // (the place that is filled next has been read)
      if (pending < STAGES) issue();
      if (pending == STAGES) asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
      else asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
      uint8_t* tile = ring + read;
      read ^= T::BYTES;
      --pending;

      // scores; x[u][0], x[u][1]: of key t0 + 16u + key_of(g), rows 2c and 2c + 1 (QUAD: twice row c); x[u][2], x[u][3]: 8
      // keys further
      float x[HALVES][4];
      {
        constexpr int W = DP / 32;                 // words of a lane's row, two steps of 16 channels each
        uint32_t wk[HALVES][2][W], sk[HALVES][2][DP / 64];
#pragma unroll
        for (int u = 0; u < HALVES; ++u)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = 16 * u + 8 * i;
            if constexpr (DP == 128) {
              const uint4 y = *reinterpret_cast<const uint4*>(tile + at_k + row * T::ROW);
              wk[u][i][0] = y.x; wk[u][i][1] = y.y; wk[u][i][W - 2] = y.z; wk[u][i][W - 1] = y.w;
            } else {
              const uint2 y = *reinterpret_cast<const uint2*>(tile + at_k + row * T::ROW);
              wk[u][i][0] = y.x; wk[u][i][1] = y.y;
            }
#pragma unroll
            for (int j = 0; j < DP / 64; ++j) sk[u][i][j] = tile[at_ks + row * T::SROW + j] * there[j];
          }
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
          for (int u = 0; u < HALVES; ++u) {
            uint32_t y[4], z[4];
            from_codes(wk[u][0][w], y);
            from_codes(wk[u][1][w], z);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              y[i] = mul_f16(y[i], sk[u][0][w / 2]);
              z[i] = mul_f16(z[i], sk[u][1][w / 2]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t k4[4] = {y[2 * i], z[2 * i], y[2 * i + 1], z[2 * i + 1]};
              if (w == 0 && i == 0) mma_first(x[u], k4, qf[0][0][0], qf[0][0][1]);
              else mma(x[u], k4, qf[0][2 * w + i][0], qf[0][2 * w + i][1]);
              if constexpr (TERMS == 2) mma(x[u], k4, qf[TERMS - 1][2 * w + i][0], qf[TERMS - 1][2 * w + i][1]);
            }
          }
      }
      if (t0 + STEP > low) {
        // (values that some row does not see: weights of 0 shall meet numbers, whatever the bytes)
        if (lane < STEP) {
          uint32_t* vs = reinterpret_cast<uint32_t*>(tile + VALUES + T::CODES + lane * T::SROW);
#pragma unroll
          for (int i = 0; i < T::SROW / 4; ++i) vs[i] = __vminu4(vs[i], SCALE_TOP * 0x01010101u);
        }
        __syncwarp();
        const int key = t0 + key_of(g);
        int lim[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) lim[r] = __shfl_sync(FULL_MASK, see, 4 * (2 * c + r));
#pragma unroll
        for (int u = 0; u < HALVES; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (key + 16 * u + (i < 2 ? 0 : 8) >= lim[i & 1]) x[u][i] = -INFINITY;
      }
      float t[R];
      bool over = false;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        t[r] = fmaxf(x[0][r], x[0][2 + r]);
#pragma unroll
        for (int u = 1; u < HALVES; ++u) t[r] = fmaxf(t[r], fmaxf(x[u][r], x[u][2 + r]));
        t[r] *= row_scale[r];
        over |= t[r] > above[r];
      }
      if (__any_sync(FULL_MASK, over)) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float top = t[r];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, d));
          // (each row by its own scores: its bits do not hang on its neighbours')
          if (top > above[r]) {
            const float alpha = ex2(above[r] - LAZY - top);
            above[r] = top + LAZY;
            less[r] = SHIFT - top;
            l[r] *= alpha;
#pragma unroll
            for (int i = 0; i < OT; ++i)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (QUAD || (k & 1) == r) o[i][k] *= alpha;
          }
        }
      }
      uint32_t pb[HALVES][TERMS][2];               // of the first and the second eight keys
#pragma unroll
      for (int u = 0; u < HALVES; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float e[R];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            e[r] = ex2(fmaf(x[u][2 * i + r], row_scale[r], less[r]));
            l[r] += e[r];
          }
          const uint32_t h = half2_of(e[0], e[R - 1]);
          pb[u][0][i] = transposed(h);
          if constexpr (TERMS == 2) {
            const float2 z = floats_of(h);
            pb[u][TERMS - 1][i] = transposed(half2_of(e[0] - z.x, e[R - 1] - z.y));
          }
        }
      // values: channels (DP / 8) g .. of keys key_of(2c), key_of(2c + 1) and 8 more each
#pragma unroll
      for (int u = 0; u < HALVES; ++u) {
        uint32_t w0[DP / 64], w1[DP / 64], w2[DP / 64], w3[DP / 64];
        auto get = [&](int at, uint32_t (&w)[DP / 64]) {
          if constexpr (DP == 128) {
            const uint2 y = *reinterpret_cast<const uint2*>(tile + at);
            w[0] = y.x;
            w[DP / 64 - 1] = y.y;
          } else {
            w[0] = *reinterpret_cast<const uint32_t*>(tile + at);
          }
        };
        const int row = 16 * u * T::ROW, row8 = row + 8 * T::ROW, srow = 16 * u * T::SROW, srow8 = srow + 8 * T::SROW;
        get(at_v[0] + row, w0);
        get(at_v[1] + row, w1);
        get(at_v[0] + row8, w2);
        get(at_v[1] + row8, w3);
        if constexpr (QUAD) {
          // A product takes eight keys: a column is a row and one of the two codes of a byte, a weight meets the one and
          // a zero the other, so that the codes of a key are converted as they lie.
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t s0 = scale_plain(tile[at_vs[0] + (i ? srow8 : srow)]), s1 = scale_plain(tile[at_vs[1] + (i ? srow8 : srow)]);
            const uint32_t b0 = __byte_perm(pb[u][0][i], 0, pick[0]), b1 = __byte_perm(pb[u][0][i], 0, pick[1]);
#pragma unroll
            for (int w = 0; w < DP / 64; ++w) {
              uint32_t y[4], z[4];
              from_codes(i ? w2[w] : w0[w], y);
              from_codes(i ? w3[w] : w1[w], z);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                y[k] = mul_f16(y[k], s0);
                z[k] = mul_f16(z[k], s1);
              }
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint32_t v4[4] = {y[2 * k], y[2 * k + 1], z[2 * k], z[2 * k + 1]};
                mma(o[2 * w + k], v4, b0, b1);
              }
            }
          }
          continue;
        }
        const uint32_t s0 = scales_plain(tile[at_vs[0] + srow], tile[at_vs[1] + srow]);
        const uint32_t s1 = scales_plain(tile[at_vs[0] + srow8], tile[at_vs[1] + srow8]);
#pragma unroll
        for (int w = 0; w < DP / 64; ++w) {        // a word: eight channels
          uint32_t ev[4], od[4], ev8[4], od8[4];   // even and odd channels of the keys' pairs
          from_codes((w0[w] & 0x0f0f0f0fu) | ((w1[w] << 4) & 0xf0f0f0f0u), ev);
          from_codes(((w0[w] >> 4) & 0x0f0f0f0fu) | (w1[w] & 0xf0f0f0f0u), od);
          from_codes((w2[w] & 0x0f0f0f0fu) | ((w3[w] << 4) & 0xf0f0f0f0u), ev8);
          from_codes(((w2[w] >> 4) & 0x0f0f0f0fu) | (w3[w] & 0xf0f0f0f0u), od8);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t v4[4] = {mul_f16(ev[i], s0), mul_f16(od[i], s0), mul_f16(ev8[i], s1), mul_f16(od8[i], s1)};
            if constexpr (TERMS == 2) {            // (these keys' sums, to be added in fp32)
              float d[4];
              mma_first(d, v4, pb[u][TERMS - 1][0], pb[u][TERMS - 1][1]);
              mma(d, v4, pb[u][0][0], pb[u][0][1]);
#pragma unroll
              for (int k = 0; k < 4; ++k) o[(4 * w + i) % OT][k] += d[k];
            } else {
              mma(o[(4 * w + i) % OT], v4, pb[u][0][0], pb[u][0][1]);
            }
          }
        }
      }
    }

    // the warps' parts meet; o[i]: channels (DP / 8) g + 2i and 2i + 1 of rows 2c and 2c + 1, or four from 4i on of row c
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[r] += __shfl_xor_sync(FULL_MASK, l[r], d);
      if (g == 0) sm.ml[warp][R * c + r] = make_float2(above[r] == -INFINITY ? -INFINITY : -less[r], l[r]);
      float* to = &sm.sums[warp][R * c + r][(DP / 8) * g];
#pragma unroll
      for (int i = 0; i < DP / 8; i += 4)
        store4(to + i, QUAD ? make_float4(o[i / 4][0], o[i / 4][1], o[i / 4][2], o[i / 4][3])
                            : make_float4(o[i / 2 % OT][r], o[i / 2 % OT][2 + r], o[(i / 2 + 1) % OT][r], o[(i / 2 + 1) % OT][2 + r]));
    }
    meet();
#pragma unroll 1
    for (int e = turn * 32 + lane; e < ROWS * (DP / 4); e += 32 * group) {
      const int r = e % ROWS, c0 = 4 * (e / ROWS);
      if (r >= f.rows || c0 >= D) continue;
      float top = -INFINITY, all = 0.f;
      for (int w = sub; w < WARPS; w += heads) top = fmaxf(top, sm.ml[w][r].x);
      const float ms = top == -INFINITY ? 0.f : top;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = sub; w < WARPS; w += heads) {
        const float2 ml = sm.ml[w][r];
        const float by = ml.x == top ? 1.f : ex2(ml.x - ms);
        all += by * ml.y;
        const float4 y = load4(&sm.sums[w][r][c0]);
        v.x = fmaf(by, y.x, v.x);
        v.y = fmaf(by, y.y, v.y);
        v.z = fmaf(by, y.z, v.z);
        v.w = fmaf(by, y.w, v.w);
      }
      if (f.whole) {
        int token, head;
        row_of(a, f, r, token, head);
        const long long row = (long long)token * (a.Hkv * a.G) + head;
        const bool none = all == 0.f || row_idle(a, token);
        const float inv = none ? 0.f : 1.f / all;
        const float4 y = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        if constexpr (TERMS == 1) store4(static_cast<__nv_bfloat16*>(a.out) + row * D + c0, y);
        else store4(static_cast<float*>(a.out) + row * D + c0, y);
        if (a.lse && c0 == 0) a.lse[row] = none ? -INFINITY : (top + log2f(all)) * (1.f / LOG2E);
      } else {
        const int per = min(PACKED_ROWS, plan.LG);
        const long long slot = (long long)sub * a.sh.slots_o + f.slot;
        store4(a.part_o + part_at(slot, per, D, r, c0), v);
        if (c0 == 0) a.ml_o[slot * per + r] = make_float2(top, all);
      }
    }
    meet();
    ++done;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T>
cudaError_t run(const PackedArgs& p, cudaStream_t stream) {
  auto kernel = packed_few_kernel<T>;
  constexpr size_t smem = sizeof(Smem<T>);
  cudaError_t e = set_up_kernel(kernel, CARVEOUT_FULL_KB, smem);
  return e != cudaSuccess ? e : launch_early(kernel, p.a.sh.grid_o, THREADS, smem, stream, false, p);
}

}  // namespace

cudaError_t launch_packed_few(const PackedArgs& p, cudaStream_t stream) {
  const bool wide = p.a.D > 64;
  if (p.a.dt != BRISK_DT_BF16) return wide ? run<Form<128, 2, false>>(p, stream) : run<Form<64, 2, false>>(p, stream);
  if (p.a.L * p.a.G <= PACKED_QUAD) return wide ? run<Form<128, 1, true>>(p, stream) : run<Form<64, 1, true>>(p, stream);
  return wide ? run<Form<128, 1, false>>(p, stream) : run<Form<64, 1, false>>(p, stream);
}

}  // namespace brisk
