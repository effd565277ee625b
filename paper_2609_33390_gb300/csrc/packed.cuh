// A context cache in 4 bits: its format, and the arguments of the calls that write, read and attend over it.
//
// A row, the D channels of an entry and key head, is D / 16 groups of 16 channels. A group has a scale s, a byte that
// holds bits 14 to 7 of a positive fp16 number (5 bits of exponent, 3 of the significand), and a channel a code of
// the e2m1 type, two a byte, the even channel low: a sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6. The channel's value is
// code times s. Such a product has at most six significant bits and lies between 2^-18 and 61440, so it is exact in
// fp16 and in bf16: what the tensor cores multiply is the value itself.
// A row's scales take 4 bytes (up to 64 channels) or 8, so that they move as one aligned word.
#pragma once

#include <cuda_fp16.h>

#include "cache.cuh"
#include "tensor_core.cuh"

namespace brisk {

constexpr int GROUP = 16;                          // channels of a scale
constexpr float SCALE_MIN = 6.103515625e-05f;      // 2^-14: the smallest normal fp16 number
constexpr float SCALE_MAX = 10240.f;               // six times it is the largest such product that fp16 holds
constexpr uint32_t SCALE_TOP = 226;                // its byte; larger ones, which no call writes, stand for it too
inline __host__ __device__ int scale_row(int D) { return D <= 64 ? 4 : 8; }

struct PackedView {   // row (s, t, h) at codes + s*seq + t*tok + h*head, its scales at scales + s*sseq + ..., in bytes
  uint8_t *codes, *scales;
  long long seq, head, sseq, shead;
  uint32_t tok, stok;
};

// x / s, correctly rounded, from r = 1 / s correctly rounded: Markstein, "Computation of elementary functions on the
// IBM RISC System/6000 processor", IBM J. Res. Dev. 34 (1990).
__device__ __forceinline__ float quotient(float x, float s, float r) {
  const float q = x * r;
  return fmaf(fmaf(-q, s, x), r, q);
}
// 1 / s of a scale: the approximate reciprocal and a Newton step, which make the correctly rounded one of all 219.
__device__ __forceinline__ float reciprocal(float s) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
  return fmaf(fmaf(-s, r, 1.f), r, r);
}
// 1 / s of a scale, rounded upwards: the Newton step's sum, rounded so, misses 1 / s by the approximation's error squared,
// 2^-45, and no 1 / s but a power of two, where the error is none, lies so near a number of fp32.
__device__ __forceinline__ float reciprocal_above(float s) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
  return __fmaf_ru(fmaf(-s, r, 1.f), r, r);
}
// The codes of numbers q, nearest, ties to the even code, saturated; the first lowest.
template <int N>
__device__ __forceinline__ uint32_t nearest_codes(const float (&q)[N]) {
  uint32_t put;
  if constexpr (N == 8)
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}" : "=r"(put)
        : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[N - 4]), "f"(q[N - 3]), "f"(q[N - 2]), "f"(q[N - 1]));
  else
    asm("{\n\t.reg .b8 a, b, z;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "mov.b32 %0, {a, b, a, b};\n\t}" : "=r"(put) : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]));
  return put;
}
// The codes of channels x / s. The exact quotient decides which is nearest.
// fp32: a tie is a quotient of few bits, which `quotient` gives exactly, and no other one is rounded to it. Negated
// quotients are taken, with which a zero's sign outlasts the correction, and the codes' signs turned.
// bf16: 8 bits over 4 differ from a tie, if at all, by 2^-11 of it, so one product decides, if it gives ties exactly: by
// 1 / s from above, cut off. (All 256 significands over all 8, on the host; one product to nearest misses some ties.)
template <typename T, int N>
__device__ __forceinline__ uint32_t codes_of(const float (&x)[N], float s) {
  constexpr bool NARROW = sizeof(T) == 2;
  const float r = NARROW ? reciprocal_above(s) : reciprocal(s);
  const f32x2 s2 = pack2(s, s), r2 = NARROW ? pack2(r, r) : pack2(-r, -r);
  float q[N];
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const f32x2 y = pack2(x[i], x[i + 1]);
    if constexpr (NARROW) {
      unpack2(mul2_cut(y, r2), q[i], q[i + 1]);
    } else {
      const f32x2 z = mul2(y, r2);
      unpack2(fma2(fma2(z, s2, y), r2, z), q[i], q[i + 1]);
    }
  }
  return NARROW ? nearest_codes(q) : nearest_codes(q) ^ 0x88888888u;
}
// The scale of a group whose largest magnitude is `top` (finite): top / 6, to nearest of 4 significant bits, as its
// byte. The quotient's own rounding never moves it onto or across a border: where top differs from a border's
// six-fold, which is exact, it differs by a unit in its last place, and that is more than half a one of the quotient.
// (bf16: a product with 1 / 6 gives the same of every top.)
template <typename T>
__device__ __forceinline__ uint32_t scale_byte(float top) {
  const float sixth = sizeof(T) == 2 ? top * (1.f / 6.f) : quotient(top, 6.f, 1.f / 6.f);
  const uint32_t b = __float_as_uint(fminf(fmaxf(sixth, SCALE_MIN), SCALE_MAX));
  return ((b + 0x7ffffu + ((b >> 20) & 1)) >> 20) - (112u << 3);
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float((byte + (112u << 3)) << 20); }   // (byte >= 8)

// The four pairs of codes of a word's bytes, as fp16 (a byte's low code in the low half).
__device__ __forceinline__ void from_codes(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// Two scales as fp16, and one twice. Products, not shifts: beside the conversions of codes, which take the units of integer
// logic two cycles each, those of multiplication have room.
__device__ __forceinline__ uint32_t scales_plain(uint32_t low, uint32_t high) { return low * 0x80u + high * 0x800000u; }
constexpr uint32_t SCALE_PLAIN = 0x800080;
__device__ __forceinline__ uint32_t scale_plain(uint32_t byte) { return byte * SCALE_PLAIN; }
// At most SCALE_MAX whatever the byte holds (the minimum takes a number before a NaN).
__device__ __forceinline__ uint32_t scale_f16(uint32_t byte) {
  uint32_t r;
  asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(scale_plain(byte)), "r"(0x71007100u));
  return r;
}
__device__ __forceinline__ uint32_t mul_f16(uint32_t x, uint32_t y) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
  return r;
}

// A row of queries whose largest magnitude has the bits `top` goes to the tensor cores times 2^up, as fp16 with a largest
// magnitude of 2^14 to 2^15; its scores are then multiplied by query_scale. (Zeros, infinities and NaN stay what they
// are. A scale too small for fp32 is the smallest number, with which -inf stays -inf.)
__device__ __forceinline__ int query_shift(uint32_t top) { return min(max(14 + 127 - (int)(top >> 23), -126), 126); }
__device__ __forceinline__ float exp2_of(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ float query_scale(float sl2, int up) {
  return fminf(fmaxf(sl2 * exp2_of(-up), 1.40129846e-45f), 3.4e38f);
}

// Writing and reading back: rows t < count[b] of T, at places start[b] + t of a cache of room S.
struct PackedMoveArgs {
  int B, T, Hkv, D, S, dt;
  Divisor by_token, by_row;          // pieces of 16 unquantised bytes of a token, and of a row
  int step;                          // tokens that a CTA's threads have at once
  CacheView k, v;                    // [B, T, Hkv, D]
  PackedView kp, vp;
  const int32_t *start, *count;      // count: nullptr for T each
  int32_t* status;
  int alone;                         // the only CTA writes the status itself
};
cudaError_t launch_packed_store(const PackedMoveArgs& a, cudaStream_t stream);
cudaError_t launch_packed_load(const PackedMoveArgs& a, cudaStream_t stream);

// Attention: a.ko and a.vo are unused.
struct PackedArgs {
  AttendArgs a;
  PackedView k, v;
};
constexpr int PACKED_ROWS = 8;       // query rows of a tile of the kernel for few
constexpr int PACKED_CTAS = 2 * CACHE_SMS;
constexpr int PACKED_WARPS = 8;
// bf16: from more rows a sequence and key head on, the kernel for many. Its tile costs the same for 1 to 128 rows, the other
// kernel reads a key again for every 8, which costs half with 64 channels (us, for many | for few; 32 heads on 8, no prefix):
//   rows of 128 channels                    12            16            20            32            128
//   1 sequence, 2000 entries           16.5 | 14.5   16.5 | 14.5   16.7 | 16.6   16.6 | 18.6   18.9 | 24.7
//   16 of 500 to 1000                  25.3 | 26.8   25.0 | 24.9   25.6 | 30.9   25.3 | 33.9   31.8 | 67.7
//   128 of 500 to 1000                 88.7 | 69.8   88.3 | 68.0   90.9 | 89.7   92.5 | 114    114  | 381
//   32 of 4000 to 8000                               99.9 | 98.6    101 | 135                  122  | 610
//   rows of 64 channels                     16            24            32            40            48
//   1 sequence, 2000 entries           14.4 | 12.4   15.0 | 14.4   14.6 | 14.7   16.3 | 14.8   16.5 | 15.4
//   16 of 500 to 1000                  21.7 | 18.6   22.6 | 24.0   21.1 | 24.6   22.7 | 24.9   22.6 | 26.7
//   128 of 500 to 1000                 67.5 | 41.2   68.8 | 54.8   68.0 | 66.0   76.9 | 78.7   77.1 | 92.2
//   189 of 200 to 400                  66.7 | 35.0   68.0 | 45.4   68.8 | 55.5   76.9 | 65.9   76.3 | 76.1
// (80 channels behave as 128: 128 sequences 77 | 82 with 12 rows, 78 | 111 with 20. 16 to 48 channels nearly as 64, with 24 rows
// and 32: 1 sequence 12 | 11 and 12 | 13, 16 sequences 18 to 19 | 19 to 21 and 18 to 19 | 21 to 22, 128 sequences 63 to 68 |
// 54 to 62 and 62 to 66 | 68 to 78, 189 short ones 63 to 67 | 42 to 47 and 62 to 67 | 53 to 59.)
inline int packed_many(int D) { return D <= 64 ? 32 : 16; }
// bf16: up to as many rows, the kernel for few has a form of its own (single tokens of 4 query heads a key head: 256
// sequences of 512 to 2048 entries over 2048 shared 115 us without it, 104 with; one of 130001 47.5 and 43.4).
constexpr int PACKED_QUAD = 4;
// Parts of a row, about, that units of several heads may lead to. In token order such units read whole lines of
// a cache (64 sequences: 1.7 times the bytes without), but divide fewer items over the CTAs, into more parts to
// join (us, single tokens; units of several heads with up to 64 parts | never | always):
//   token order  1 of 30000: 22.7 | 22.8 | 30.5   1 of 4000: 14.3 | 14.5 | 18.6   64 of 4000: 61.9 | 81.5 | 61.9
//                64 of 500:  22.8 | 26.7 | 22.7   8 of 4000: 22.0 | 22.6 | 21.5
//   head order   1 of 30000: 21.6 | 21.5 | 28.8   64 of 4000: 55.8 | 58.9 | 55.9
constexpr int PACKED_PARTS = 64;
// The kernel for few rows: a unit is the keys of several neighbouring heads, a head a warp or several warps a head, as many
// heads as there are warps, while that leaves a row about PACKED_PARTS parts to join.
inline void divide_packed(AttendArgs* a) {
  const bool tc = a->dt == BRISK_DT_BF16, many = tc && a->L * a->G > packed_many(a->D);
  a->sh.kt = tc ? TC_KT : SIMT_KT;                 // (the prefix's)
  a->sh.rt_o = many ? SLOT_ROWS : PACKED_ROWS;
  // (bf16: tiles of 256 rows also where there are fewer. One sequence's rows behind a prefix alone, us, and with tiles of 128 in one
  // launch, as prefix and own entries in bf16 have it: 4 rows over 2048 entries 14.4 | 11.5, over 32768 41.5 | 33.1, over
  // 131072 101 | 90; 128 rows over 2048 16.9 | 14.6, over 32768 42.8 | 41.8.)
  a->sh.rt_p = tc ? PAIR_ROWS : SIMT_ROWS;
  a->sh.grid_p = a->P == 0 ? 0 : (tc ? CACHE_SMS : SLOT_CTAS);
  a->joins = tc;
  a->sh.grid_o = PACKED_CTAS;
  a->sh.weight = 1;
  a->sh.set(a->B, a->L * a->G, a->P);
  const long long items = (long long)a->B * a->Hkv * a->sh.nLT;
  int log_heads = 0;
  while (!many && (2 << log_heads) <= UNIT_HEADS && a->Hkv % (2 << log_heads) == 0 &&
         (long long)a->sh.grid_o * (2 << log_heads) <= PACKED_PARTS * items)
    ++log_heads;
  a->sh.log_kt = many || log_heads == 0 ? 7 : (log_heads == 1 ? 6 : 5);
  a->sh.kt = 1 << a->sh.log_kt;
  a->sh.log_heads = log_heads;
  a->sh.slots_o = (int)((items >> log_heads) + a->sh.grid_o);
}
cudaError_t launch_packed_few(const PackedArgs& p, cudaStream_t stream);
cudaError_t launch_packed_tc(const PackedArgs& p, cudaStream_t stream);

}  // namespace brisk
