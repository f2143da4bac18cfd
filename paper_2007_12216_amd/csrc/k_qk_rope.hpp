// Norms of queries and keys per head with the position rotation, to memory or on into the 4-bit cache; reading the cache back.
#pragma once
#include "cache4.hpp"

namespace rnswino {

// One pass: y = x / sqrt(mean(x^2) + eps) * w over a head's D dimensions, then the rotation of the first `rotary` of them by the
// token's angles: a' = a cos - b sin, b' = b cos + a sin, pairs (i, i + rotary / 2) or (2i, 2i + 1).  Lanes hold eight dimensions each, D / 8 lanes (of
// 8, 16 or 32) a head, so a head is one 16-byte load and store a lane; sums and partners come by shuffles within the head's lanes, and a head's 32-dimension
// blocks of the cache are four lanes.  Bound by HBM: each value is read and written once, everything else comes from the L1 (angles, weights).
// All of it is in 32 bits, products and sums rounded one by one, neighbours summed first: the codes are the same as those of the formula written in
// elementary operations of 32 bits.
struct RopeArgs {
  const void *q, *k, *v;
  void *q_out, *k_out;
  const void *wq, *wk;
  const float *angles;
  const int32_t *positions;
  const int64_t *slots;
  Cache4 cache;
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
  int32_t tokens, q_heads, kv_heads, dim, rotary, adjacent, max_position;
  float eps, inv_dim;
};

template <typename T>
__device__ __forceinline__ void unpack8(u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = T::low(w[e]);
    x[2 * e + 1] = T::high(w[e]);
  }
}
template <typename T>
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  return u32x4{T::pair(x[0], x[1]), T::pair(x[2], x[3]), T::pair(x[4], x[5]), T::pair(x[6], x[7])};
}

// PAST_CACHES: results of more than the L2s hold go past them: 8192 tokens of 40 heads of 128 44.7 -> 35.6 us, 4.8 TB/s where a copy makes 5.1.
template <typename T, int LANES, bool TO_CACHE, bool PAST_CACHES>
__global__ __launch_bounds__(256) void k_qk_rope(RopeArgs a) {
#pragma clang fp contract(off)
  constexpr int kPerBlock = 256 / LANES;
  const int heads = a.q_heads + a.kv_heads + (TO_CACHE ? a.kv_heads : 0);
  const int lane = threadIdx.x % LANES;                          // of the head's lanes
  const int item = blockIdx.x * kPerBlock + threadIdx.x / LANES;  // the host keeps the threads, LANES a head, below 2^32, so that heads are below 2^29
  const int token = item / heads, head = item - token * heads;
  const bool live = token < a.tokens && 8 * lane < a.dim;
  const bool is_q = head < a.q_heads, is_v = TO_CACHE && head >= a.q_heads + a.kv_heads;
  const int kv_head = is_v ? head - a.q_heads - a.kv_heads : head - a.q_heads;

  int position = -1;
  int64_t slot = -1;
  float x[8];
  u32x4 raw = {0, 0, 0, 0};
  if (live) {
    position = a.positions[token];
    if (TO_CACHE) slot = a.slots[token];
    const uint16_t *row = is_q   ? (const uint16_t *)a.q + token * a.q_stride + (int64_t)head * a.dim
                          : is_v ? (const uint16_t *)a.v + token * a.v_stride + (int64_t)kv_head * a.dim
                                 : (const uint16_t *)a.k + token * a.k_stride + (int64_t)kv_head * a.dim;
    raw = *(const u32x4 *)(row + 8 * lane);
  }
  unpack8<T>(raw, x);
  const bool placed = (uint32_t)position < (uint32_t)a.max_position;

  if (!is_v) {
    const void *weights = is_q ? a.wq : a.wk;
    if (weights) {
      float s[8], w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = x[e] * x[e];
      float sum = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
#pragma unroll
      for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
      const float r = 1.0f / sqrtf(sum * a.inv_dim + a.eps);
      unpack8<T>(live ? *(const u32x4 *)((const uint16_t *)weights + 8 * lane) : u32x4{0, 0, 0, 0}, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (x[e] * r) * w[e];
    }
    const bool turns = live && placed && 8 * lane < a.rotary;
    const float *row = a.angles + (int64_t)(placed ? position : 0) * a.rotary;
    if (a.adjacent) {
      if (turns) {
        const f32x4 cos = *(const f32x4 *)(row + 4 * lane), sin = *(const f32x4 *)(row + a.rotary / 2 + 4 * lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float even = x[2 * e], odd = x[2 * e + 1];
          x[2 * e] = even * cos[e] - odd * sin[e];
          x[2 * e + 1] = odd * cos[e] + even * sin[e];
        }
      }
    } else {
      const int half = a.rotary / 16;  // lanes
      const int with = lane < half ? lane + half : lane - half;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = __shfl(x[e], with & (LANES - 1), LANES);
      if (turns) {
        const int at = 8 * (lane < half ? lane : with);
        const f32x4 cos[2] = {*(const f32x4 *)(row + at), *(const f32x4 *)(row + at + 4)};
        const f32x4 sin[2] = {*(const f32x4 *)(row + a.rotary / 2 + at), *(const f32x4 *)(row + a.rotary / 2 + at + 4)};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float turned = y[e] * sin[e / 4][e % 4], kept = x[e] * cos[e / 4][e % 4];
          x[e] = lane < half ? kept - turned : kept + turned;
        }
      }
    }
    if (!placed) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0;
    }
  }

  if (!TO_CACHE || is_q) {
    if (live) {
      uint16_t *row = is_q ? (uint16_t *)a.q_out + token * a.q_out_stride + (int64_t)head * a.dim
                           : (uint16_t *)a.k_out + token * a.k_out_stride + (int64_t)kv_head * a.dim;
      if constexpr (PAST_CACHES) __builtin_nontemporal_store(pack8<T>(x), (u32x4 *)(row + 8 * lane));
      else *(u32x4 *)(row + 8 * lane) = pack8<T>(x);
    }
  }
  if constexpr (TO_CACHE) {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    most = max(most, (uint32_t)__shfl_xor((int)most, 1));
    most = max(most, (uint32_t)__shfl_xor((int)most, 2));
    if (!is_q && live && placed && slot >= 0 && slot < ((int64_t)a.cache.pages << a.cache.page_shift)) {
      const uint32_t byte = scale_byte(most);
      const int64_t row = cache_row(a.cache, slot, kv_head);
      uint8_t *codes = is_v ? a.cache.v : a.cache.k, *scales = is_v ? a.cache.v_scale : a.cache.k_scale;
      *(uint32_t *)(codes + row * (a.dim / 2) + 4 * lane) = to_codes(x, byte);
      if (lane % 4 == 0) scales[row * (a.dim / 32) + lane / 4] = (uint8_t)byte;
    }
  }
}

// The values of cached rows, [n][heads][D] for k and v each: eight dimensions a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_cache4_read(Cache4 c, const int64_t *slots, int64_t n, uint16_t *k_out, uint16_t *v_out) {
  const int per_row = c.dim / 8;
  const int64_t per_token = (int64_t)c.heads * per_row, total = n * per_token;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < 2 * total; i += (int64_t)gridDim.x * 256) {
    const bool is_v = i >= total;
    const int64_t at = is_v ? i - total : i;
    const int64_t token = at / per_token;
    const int rest = (int)(at - token * per_token), head = rest / per_row, piece = rest - head * per_row;
    const int64_t slot = slots[token];
    u32x4 out = {0, 0, 0, 0};
    if (slot >= 0 && slot < ((int64_t)c.pages << c.page_shift)) {
      const int64_t row = cache_row(c, slot, head);
      const uint32_t codes = *(const uint32_t *)((is_v ? c.v : c.k) + row * (c.dim / 2) + 4 * piece);
      const float scale = __uint_as_float((uint32_t)(is_v ? c.v_scale : c.k_scale)[row * (c.dim / 32) + piece / 4] << 23);
      const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1),
                  p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
      out = u32x4{T::pair(p0.x, p0.y), T::pair(p1.x, p1.y), T::pair(p2.x, p2.y), T::pair(p3.x, p3.y)};
    }
    *(u32x4 *)((is_v ? v_out : k_out) + at * 8) = out;
  }
}

}  // namespace rnswino
