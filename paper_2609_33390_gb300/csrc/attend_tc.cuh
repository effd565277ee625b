// Attention on the tensor cores, a slot of 128 query rows a row a thread: what the kernels over bf16 caches and over
// caches in 4 bits share (see cache_attend_tc.cu).
#pragma once

#include <cuda_fp16.h>

#include "cache.cuh"
#include "tensor_core.cuh"

namespace brisk {
namespace {

constexpr int KT = TC_KT, SLOT = SLOT_ROWS;
constexpr int PANEL = TILE_PANEL;

// The weights that enter the product with the values: LAZY is log2 of what a score may exceed the held maximum by,
// 2^SHIFT what a weight at the held maximum is. fp16 ends at 2^16, and holds 11 bits down to 2^-14.
template <typename T> struct WeightAs;
template <> struct WeightAs<__nv_bfloat16> {
  static constexpr float LAZY = 8.f, SHIFT = 0.f;
  static __device__ __forceinline__ uint32_t pair(float x, float y) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <> struct WeightAs<__half> {
  static constexpr float LAZY = 5.f, SHIFT = 10.f;
  static __device__ __forceinline__ uint32_t pair(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

// A slot's row of a thread: token * Hq + head (its complement: padding, -1: none), the keys it sees, its query.
struct Row {
  int id, lim;
  const __nv_bfloat16* q;
};

__device__ __forceinline__ Row find_row(const AttendArgs& a, const Frag& f, int row) {
  Row x{-1, f.len, nullptr};
  if (row < f.rows) {
    int token, head;
    row_of(a, f, row, token, head);
    const int b = a.by_L.of(token), i = token - b * a.L;
    x.id = token * (a.Hkv * a.G) + head;
    x.q = static_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.seq + i * a.q.tok + head * a.q.head;
    if (a.visible) {
      const int v = a.visible[token];
      if (v < 0) x.id = ~x.id;
      if (!f.prefix) x.lim = max(0, min(x.lim, v));
    }
  }
  return x;
}

__device__ __forceinline__ void rows_fetched() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  fence_async_smem();
}

// One tile of a row: from the scores at tS its weights, over them, as W has them; m and l go on, and O at tO is
// rescaled where the maximum moved (unless this is the slot's first tile). `seen`: keys of the tile that
// the row sees. half() is called when the weights of the first half of the keys are there.
template <typename W, typename Half>
__device__ __forceinline__ void row_weights(uint32_t tS, uint32_t tO, int D, int seen, float sl2, bool first, float& m,
                                            float& l, Half half) {
  float v[KT];
  tmem_ld128(tS, v);
  if (__any_sync(FULL_MASK, seen < KT)) {
#pragma unroll
    for (int c = 0; c < KT; ++c) v[c] = c < seen ? v[c] : -INFINITY;
  }
  float top[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
  for (int c = 4; c + 8 <= KT; c += 8)
#pragma unroll
    for (int i = 0; i < 4; ++i) top[i] = fmaxf(fmaxf(top[i], v[c + i]), v[c + 4 + i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) top[i] = fmaxf(top[i], v[KT - 4 + i]);
  const float t = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * sl2;
  // (each row by its own scores: a row's bits must not hang on its neighbours', of which some may be no rows at all)
  const bool over = t > m + W::LAZY;
  if (__any_sync(FULL_MASK, over)) {
    const float alpha = over ? ex2(m - t) : 1.f;   // (t is no -inf)
    if (over) m = t;
    l *= alpha;
    if (!first)
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
  const float ms = m == -INFINITY ? 0.f : m - W::SHIFT;
  const f32x2 scale2 = pack2(sl2, sl2), minus2 = pack2(-ms, -ms);
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
      p[c / 2] = W::pair(x[0], x[1]);
      p[c / 2 + 1] = W::pair(x[2], x[3]);
    }
    tmem_st16(tS + c0 / 2, p);
    if (c0 + 32 == KT / 2) {
      tmem_st_wait();
      half();
    }
  }
  float x[2];
  unpack2(add2(sum0, sum1), x[0], x[1]);
  l += x[0] + x[1];
  tmem_st_wait();
}

// The rows' end: their results, or their parts, from O at tO. `part`: column 0 of the row in the slot of
// parts, nullptr for the result, which (JOIN) the first `others.n` <= 2 parts of other keys then join. Results go
// through `stage` (2 KB a warp), so that 4 lanes write 64 bytes of a row: a row a lane, every store would touch 32
// lines.
constexpr int STAGE_BYTES = 32 * 64;
template <bool JOIN>
__device__ __forceinline__ void store_rows(const AttendArgs& a, uint32_t tO, const Row& x, bool mine, float m, float l,
                                           float* part, float2* ml, int per, uint8_t* stage, const Parts& others) {
  const int lane = threadIdx.x & 31, D = a.D;
  const int row = x.id < 0 ? ~x.id : x.id;
  float w = 1.f, w0 = 0.f, w1 = 0.f;               // weights of this part and the others
  const bool one = JOIN && mine && !part && others.n > 0, two = one && others.n > 1;
  const float* src0 = others.sums;
  const float* src1 = others.sums + (two ? others.per * D : 0);
  if (one) {
    const float2 y = others.ml[0], z = two ? others.ml[others.per] : make_float2(-INFINITY, 0.f);
    const float top = fmaxf(m, fmaxf(y.x, z.x)), ms = top == -INFINITY ? 0.f : top;
    w = m == top ? 1.f : ex2(m - ms);
    w0 = y.x == top ? 1.f : ex2(y.x - ms);
    w1 = !two ? 0.f : (z.x == top ? 1.f : ex2(z.x - ms));
    m = top;
    l = w * l + w0 * y.y + w1 * z.y;
  }
  const bool none = l == 0.f || x.id < 0;
  const float inv = none ? 0.f : 1.f / l;
  const bool direct = mine && !part;
  const int to_row = direct ? row : -1;
  const bool any_direct = __any_sync(FULL_MASK, direct);
#pragma unroll 1
  for (int c = 0; c < D; c += 32) {
    float o[32];
    if (JOIN && __any_sync(FULL_MASK, one)) {      // (all loads on their way before the first is used)
      float4 y[8], z[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int at = min(c + 4 * k, D - 4) * others.per;
        y[k] = one ? load4(src0 + at) : make_float4(0.f, 0.f, 0.f, 0.f);
        z[k] = two ? load4(src1 + at) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      tmem_ld32(tO + c, o);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        o[4 * k] = fmaf(w1, z[k].x, fmaf(w0, y[k].x, w * o[4 * k]));
        o[4 * k + 1] = fmaf(w1, z[k].y, fmaf(w0, y[k].y, w * o[4 * k + 1]));
        o[4 * k + 2] = fmaf(w1, z[k].z, fmaf(w0, y[k].z, w * o[4 * k + 2]));
        o[4 * k + 3] = fmaf(w1, z[k].w, fmaf(w0, y[k].w, w * o[4 * k + 3]));
      }
    } else {
      tmem_ld32(tO + c, o);
    }
    if (mine && part) {
#pragma unroll
      for (int i = 0; i < 32; i += 4)
        if (c + i < D) store4(part + (c + i) * per, make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]));
    }
    __syncwarp();
    if (any_direct) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {                // 16-byte pieces of the row, swizzled over its 64 bytes
        uint32_t y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const __nv_bfloat162 h = none ? __floats2bfloat162_rn(0.f, 0.f)
                                        : __floats2bfloat162_rn(o[8 * i + 2 * k] * inv, o[8 * i + 2 * k + 1] * inv);
          y[k] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(stage + lane * 64 + ((i ^ (lane >> 1)) & 3) * 16) = make_uint4(y[0], y[1], y[2], y[3]);
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 32; i += 8) {
        const int r = i + (lane >> 2), to = __shfl_sync(FULL_MASK, to_row, r), q = lane & 3;
        const uint4 y = *reinterpret_cast<const uint4*>(stage + r * 64 + ((q ^ (r >> 1)) & 3) * 16);
        if (to >= 0 && c + 8 * q < D)
          *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + (long long)to * D + c + 8 * q) = y;
      }
      __syncwarp();
    }
  }
  if (!mine) return;
  if (part) *ml = make_float2(m, l);
  else if (a.lse) a.lse[row] = none ? -INFINITY : (m + log2f(l)) * (1.f / LOG2E);
}

// The products of 128 rows with a tile, issued by one thread: scores (16 columns a step, nd of them), and
// values for steps s0 <= step < s1 of 16 keys.
template <int DP>
__device__ __forceinline__ void issue_scores(uint32_t tS, uint32_t q_lo, uint32_t k_lo, int nd, uint32_t idesc) {
#pragma unroll
  for (int kk = 0; kk < DP / 16; ++kk) {
    const uint32_t o = (kk >> 2) * (PANEL >> 4) + 2 * (kk & 3);
    if (kk < nd) umma(tS, sw128(q_lo + o), sw128(k_lo + o), idesc, kk > 0);
  }
}
template <int HALF>
__device__ __forceinline__ void issue_values(uint32_t tO, uint32_t tS, uint32_t v_lo, int steps, uint32_t idesc, bool begun) {
#pragma unroll
  for (int kk = HALF * (KT / 32); kk < (HALF + 1) * (KT / 32); ++kk)
    if (kk < steps) umma_ts(tO, tS + 8 * kk, sw128(v_lo + kk * 128), idesc, begun || kk > 0);
}

}  // namespace
}  // namespace brisk
