// Matrix products in 8-bit floating point with a scale for each block of 128, and the quantisation of their operands.
#pragma once
#include "decoder_common.hpp"

namespace rnswino {

// y[m][n] = sum over blocks b of xs[b][m] ws[n / 128][b] (sum over the block's 128 inputs of x w), x and w in e4m3 (4 bits of exponent, 3 of fraction,
// largest 448).  Rows of codes are whole blocks long; what is behind the last input is zero.
constexpr int kBlock = 128;
// Below this a block counts as this: its codes are then next to 0, and 448 / max is finite.
constexpr float kLeastMax = 0x1p-100f;

// Rows begin at any multiple of 2 bytes (39 x 161 x 1569, an element a load: 10.3 us).
typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef uint32_t u32x2_2 __attribute__((ext_vector_type(2), aligned(2), may_alias));
// Elements [at, at + 8) of a row of `cols`, zeros behind its end.
template <typename T>
__device__ __forceinline__ void load8(const uint16_t *row, int at, int cols, float (&x)[8]) {
  if (at + 8 <= cols) {
    const u32x4_2 w = *(const u32x4_2 *)(row + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[2 * e] = T::low(w[e]), x[2 * e + 1] = T::high(w[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = at + e < cols ? T::widen(row[at + e]) : 0.0f;
  }
}
__device__ __forceinline__ float most_of(const float (&x)[8]) {
  float most = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
  return most;
}
// The largest of 16 neighbouring lanes, in all of them, by moves inside the vector unit: lanes 1 and 2 apart, then mirrored in halves and in whole.
__device__ __forceinline__ float most_of_16(float x) {
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0xB1, 0xF, 0xF, true)));
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x4E, 0xF, 0xF, true)));
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x141, 0xF, 0xF, true)));
  return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x140, 0xF, 0xF, true)));
}
// To the nearest, ties to even; |x factor| <= 448 (1 + 2^-23), which rounds to 448.  NaN stays NaN, an infinity (factor 0) becomes one.
__device__ __forceinline__ u32x2 to_e4m3(const float (&x)[8], float factor) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * factor, x[1] * factor, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * factor, x[3] * factor, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * factor, x[5] * factor, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * factor, x[7] * factor, hi, true);
  return u32x2{(uint32_t)lo, (uint32_t)hi};
}

// Rows in blocks of 1 x 128: 16 lanes a block, 8 inputs each.
template <typename T>
__global__ __launch_bounds__(256) void k_fp8_rows(const uint16_t *x, int64_t stride, int rows, int cols, int blocks, uint8_t *codes, float *scales) {
  const int lane = threadIdx.x & 15;
  const int64_t items = (int64_t)rows * blocks;
  for (int64_t item = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); item < items; item += (int64_t)gridDim.x * 16) {
    const int64_t row = item / blocks;
    const int block = (int)(item - row * blocks), at = block * kBlock + 8 * lane;
    float v[8];
    load8<T>(x + row * stride, at, cols, v);
    const float most = fmaxf(most_of_16(most_of(v)), kLeastMax);
    *(u32x2 *)(codes + row * blocks * kBlock + at) = to_e4m3(v, 448.0f / most);
    if (lane == 0) scales[(int64_t)block * rows + row] = most / 448.0f;
  }
}

// Weights in blocks of 128 x 128, a workgroup each, a row of the block by 16 lanes; done once for a model, so read twice (the second time from the L2).
template <typename T>
__global__ __launch_bounds__(256) void k_fp8_weights(const uint16_t *w, int64_t stride, int rows, int cols, int blocks, uint8_t *codes, float *scales) {
  __shared__ float partial[4];
  const int lane = threadIdx.x & 15, sub = threadIdx.x >> 4, block = blockIdx.x % blocks, tall = blockIdx.x / blocks, at = block * kBlock + 8 * lane;
  float most = 0, v[8];
  for (int r = sub; r < kBlock && tall * kBlock + r < rows; r += 16) {
    load8<T>(w + (int64_t)(tall * kBlock + r) * stride, at, cols, v);
    most = fmaxf(most, most_of(v));
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
  if ((threadIdx.x & 63) == 0) partial[threadIdx.x >> 6] = most;
  __syncthreads();
  most = fmaxf(fmaxf(fmaxf(partial[0], partial[1]), fmaxf(partial[2], partial[3])), kLeastMax);
  for (int r = sub; r < kBlock && tall * kBlock + r < rows; r += 16) {
    const int64_t row = tall * kBlock + r;
    load8<T>(w + row * stride, at, cols, v);
    *(u32x2 *)(codes + row * blocks * kBlock + at) = to_e4m3(v, 448.0f / most);
  }
  if (threadIdx.x == 0) scales[(int64_t)tall * blocks + block] = most / 448.0f;
}

typedef int v8i __attribute__((ext_vector_type(8)));
// One block of 128 inputs: rows of `w` by columns of `x`, from zero (the operands' blocks have scales of their own, applied to the sum).  The instruction adds products by eights first, and
// there cuts what lies below 2^-13 of the largest (measured: beside 2^16 and -2^16 a product of 2^3 is kept and one of 2^2 lost; between the eights 2^-24).  That is the accuracy of the
// matrix cores with this type, taken since a code's own rounding is 2^-4 of it; sums over blocks, and scales, are in 32 bits.
__device__ __forceinline__ f32x4 block_product(u32x4 w0, u32x4 w1, u32x4 x0, u32x4 x1) {
  const v8i w = {(int)w0.x, (int)w0.y, (int)w0.z, (int)w0.w, (int)w1.x, (int)w1.y, (int)w1.z, (int)w1.w};
  const v8i x = {(int)x0.x, (int)x0.y, (int)x0.z, (int)x0.w, (int)x1.x, (int)x1.y, (int)x1.z, (int)x1.w};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}

struct Fp8Args {
  const uint8_t *x, *w;  // x: codes, or rows of 16-bit elements x_stride apart
  const float *xs, *ws;
  uint16_t *y;
  int64_t y_stride, x_stride;
  int32_t rows, outputs, blocks, inputs;
};

// Four outputs of one row, the first `there` of them in range.
template <typename T>
__device__ __forceinline__ void store4(uint16_t *to, f32x4 v, int there) {
  if (there >= 4) {
    *(u32x2_2 *)to = u32x2_2{T::pair(v[0], v[1]), T::pair(v[2], v[3])};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < there) to[i] = T::one(v[i]);
  }
}

// 16 bytes a lane from memory into LDS: lane i's land at `to` + 16 i.
__device__ __forceinline__ void load_to_lds(const uint8_t *from, uint8_t *to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// A float a lane.
__device__ __forceinline__ void scale_to_lds(const float *from, uint8_t *to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 4, 0, 0);
}

// Workgroup ids go to the 8 XCDs in turn, and each has an L2 of its own: XCD i gets the i-th eighth of the tiles, in bands of 8 tiles of rows, an output tile after another, so that
// what runs together shares rows and weights.  `id` runs to a multiple of 8; false behind the last tile.
struct TileAt {
  int n, m;
};
__device__ __forceinline__ bool tile_at(int id, int tiles_n, int tiles_m, TileAt &at) {
  const int tiles = tiles_n * tiles_m, item = (id & 7) * ((tiles + 7) >> 3) + (id >> 3);
  if (item >= tiles || (id >> 3) >= ((tiles + 7) >> 3)) return false;
  const int band = item / (8 * tiles_n), in_band = item - band * 8 * tiles_n, tall = min(8, tiles_m - 8 * band);
  at = {in_band / tall, 8 * band + in_band % tall};
  return true;
}

// Until at most N of this wave's loads are under way, and no reads of LDS.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");  // (the waitcnt alone orders nothing for the compiler)
  __builtin_amdgcn_s_waitcnt((N & 15) | 0x0070 | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}

// Many rows: a workgroup of WN x WM waves, each of RN x RM products of 16 outputs x 16 rows, takes a block of inputs a step, both operands through STAGES stages of LDS that are
// filled without passing registers, STAGES - 1 blocks ahead.  The weights are the products' rows, so a lane holds four neighbouring outputs of one row of y, and one scale.
// Bound by the matrix cores, and then by LDS: a wave reads 16 (RN + RM) rows of 128 bytes for RN RM products of 32 cycles.
template <typename T, int WN, int WM, int RN, int RM, int STAGES>
__global__ __launch_bounds__(64 * WN * WM, 2) void k_fp8_many(Fp8Args a) {
  constexpr int kWaves = WN * WM, kN = 16 * WN * RN, kM = 16 * WM * RM, kPieces = (kN + kM) / 8 / kWaves, kLoads = kPieces + 2;
  constexpr int kScales = (kN + kM) * kBlock, kStage = kScales + kWaves * 512;  // a wave's scales: 64 of rows, then one of the weights, 64 times
  static_assert((kN + kM) / 8 % kWaves == 0 && kN / 8 % kWaves == 0, "a wave's loads are eight rows of one operand each");
  static_assert(128 % (16 * RN) == 0 && RM <= 4, "a wave's outputs lie under one scale of the weights, its rows under one load of scales");
  __shared__ __align__(16) uint8_t stages[STAGES * kStage];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  TileAt at;
  if (!tile_at(blockIdx.x, (a.outputs + kN - 1) / kN, (a.rows + kM - 1) / kM, at)) return;
  const int n0 = at.n * kN, m0 = at.m * kM, wn = (wave % WN) * 16 * RN, wm = (wave / WN) * 16 * RM;
  const int64_t pitch = (int64_t)a.blocks * kBlock;

  // 16-byte pieces of a row of a block lie in LDS in the order piece ^ (row / 2 % 8), and a lane reads pieces g and g + 4 of a row (of both operands: the contraction's order is free): with
  // that a read takes 4 cycles, with pieces 2g and 2g + 1, or in order, 8
  const uint8_t *from[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int row = (i * kWaves + wave) * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
    from[i] = (i < kN / 8 / kWaves ? a.w + min(n0 + row, a.outputs - 1) * pitch : a.x + min(m0 + row - kN, a.rows - 1) * pitch) + 16 * piece;
  }
  const float *xs = a.xs + min(m0 + wm + lane, a.rows - 1), *ws = a.ws + (int64_t)min((n0 + wn) / kBlock, (a.outputs - 1) / kBlock) * a.blocks;
  int fetched = 0;
  const auto fetch = [&](int to) {
    uint8_t *const stage = stages + to * kStage;
    scale_to_lds(xs, stage + kScales + wave * 512);
    scale_to_lds(ws, stage + kScales + wave * 512 + 256);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) load_to_lds(from[i], stage + (i * kWaves + wave) * 1024);
    const int more = ++fetched < a.blocks;  // behind the last block that one again, so that the loads under way are always as many
    xs += more ? a.rows : 0, ws += more;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) from[i] += more ? kBlock : 0;
  };
  f32x4 sum[RN][RM];
#pragma unroll
  for (int i = 0; i < RN; ++i)
#pragma unroll
    for (int j = 0; j < RM; ++j) sum[i][j] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) fetch(s);
  int now = 0;
  for (int block = 0; block < a.blocks; ++block) {
    // this wave's part of the stage that is read now has arrived, and it has read the one before: behind the barrier so have all
    wait_loads<kLoads *(STAGES - 2)>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    const uint8_t *const read = stages + now * kStage;
    const float *const scales = (const float *)(read + kScales + wave * 512);
    float scale[RM];
#pragma unroll
    for (int j = 0; j < RM; ++j) scale[j] = scales[16 * j + r] * scales[64];
    const auto operand = [&](int row, u32x4 (&to)[2]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) to[h] = *(const u32x4 *)(read + row * kBlock + 16 * ((g + 4 * h) ^ (r >> 1)));
    };
    // A product, and beside it the sums of the one before: their scales are the block's, so they cannot be left to the next product.  (In the compiler's own order a product is waited for, 12
    // wait states, before its sums, and the next one begins after them: 29 % of the matrix cores' cycles.)
    u32x4 x[RM][2], w[2][2];
    f32x4 before[RM];
    operand(wn + r, w[0]);
#pragma unroll
    for (int j = 0; j < RM; ++j) operand(kN + wm + 16 * j + r, x[j]);
#pragma unroll
    for (int i = 0; i < RN; ++i) {
      if (i + 1 < RN) operand(wn + 16 * (i + 1) + r, w[(i + 1) & 1]);
      if (i == 0) {  // behind the first reads, which would wait for the loads' addresses to be taken
        __builtin_amdgcn_sched_barrier(0);
        fetch(now == 0 ? STAGES - 1 : now - 1);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < RM; ++j) {
        const f32x4 product = block_product(w[i & 1][0], w[i & 1][1], x[j][0], x[j][1]);
        if (i) sum[i - 1][j] += before[j] * scale[j];
        before[j] = product;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int j = 0; j < RM; ++j) sum[RN - 1][j] += before[j] * scale[j];
    now = now == STAGES - 1 ? 0 : now + 1;
  }
  wait_loads<0>();
#pragma unroll
  for (int j = 0; j < RM; ++j) {
    const int row = m0 + wm + 16 * j + r;
    if (row >= a.rows) continue;
#pragma unroll
    for (int i = 0; i < RN; ++i) {
      const int n = n0 + wn + 16 * i + 4 * g;
      store4<T>(a.y + row * a.y_stride + n, sum[i][j], a.outputs - n);
    }
  }
}

// Few rows: a workgroup computes 16 outputs x 16 COLS rows; its waves take the blocks of inputs in turn, each through STAGES stages of LDS of its own (a wave's loads that go straight to
// the operands' registers have 16 rows in neighbouring lanes, 42 accesses of the L1 each instead of 16: 203 x 1000 x 4600 in 17 us), and add up in LDS in the waves' order.  Bound by the
// weights' bytes, and by what a step waits for: as built, a step first waits for all loads under way (its scales, which come through registers, are behind the stages' first loads, and loads are
// counted in order), so the stages are filled ahead of the loop and by one block a step behind that.  FROM_ROWS: x is 16-bit rows, of which each workgroup quantises its own into LDS (kFewCodes
// at most) by itself, which is less than a launch, and two stages leave room for three workgroups on a compute unit (8192 x 2048, 1 row: four stages, one workgroup, 10.5 us; two 8.1).  There
// the compiler waits for the block that has just been asked for too, before operands are read: it cannot tell the LDS that they are read from from the LDS that is being filled.
constexpr int kFewCodes = 16384;

template <typename T, int COLS, bool FROM_ROWS, int WAVES, int STAGES>
__global__ __launch_bounds__(64 * WAVES) void k_fp8_few(Fp8Args a) {
  constexpr int kRows = FROM_ROWS ? 16 : 16 + 16 * COLS, kLoads = kRows / 8, kStage = kRows * kBlock;
  __shared__ __align__(16) uint8_t lds[WAVES * STAGES * kStage];
  __shared__ __align__(16) uint8_t x_codes[FROM_ROWS ? kFewCodes : 16];
  __shared__ float x_scales[FROM_ROWS ? kFewCodes / kBlock : 1];  // [block][row]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * COLS;
  const int held = min(16 * COLS, a.rows - m0);  // rows that there are
  const int64_t pitch = (int64_t)a.blocks * kBlock;
  uint8_t *const mine = lds + wave * STAGES * kStage;

  // as in k_fp8_many, eight rows a load
  const uint8_t *from[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = 8 * i + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
    from[i] = (i < 2 ? a.w + min(n0 + row, a.outputs - 1) * pitch : a.x + min(m0 + row - 16, a.rows - 1) * pitch) + 16 * piece;
  }
  const auto fetch = [&](int block, int to) {  // behind the last block: that one again, so that the loads under way are always as many
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_to_lds(from[i] + (int64_t)min(block, a.blocks - 1) * kBlock, mine + to * kStage + i * 1024);
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) fetch(wave + s * WAVES, s);
  if constexpr (FROM_ROWS) {
    const int items = held * a.blocks, lane16 = threadIdx.x & 15;
    const int row_step = 4 * WAVES / a.blocks, block_step = 4 * WAVES - row_step * a.blocks;
    int row = (int)(threadIdx.x >> 4) / a.blocks, block = (int)(threadIdx.x >> 4) - row * a.blocks;
    for (int item = threadIdx.x >> 4; item < items; item += 4 * WAVES) {
      const int at = block * kBlock + 8 * lane16;
      float v[8];
      load8<T>((const uint16_t *)a.x + (m0 + row) * a.x_stride, at, a.inputs, v);
      const float most = fmaxf(most_of_16(most_of(v)), kLeastMax);
      *(u32x2 *)(x_codes + item * kBlock + 8 * lane16) = to_e4m3(v, 448.0f / most);
      if (lane16 == 0) x_scales[block * held + row] = most / 448.0f;
      row += row_step, block += block_step;
      if (block >= a.blocks) ++row, block -= a.blocks;
    }
    __syncthreads();
  }
  const float *ws = a.ws + (int64_t)(n0 / kBlock) * a.blocks;
  int m[COLS];
  f32x4 sum[COLS];
#pragma unroll
  for (int j = 0; j < COLS; ++j) {
    m[j] = min(16 * j + r, held - 1);
    sum[j] = f32x4{0, 0, 0, 0};
  }
  float next[COLS], next_ws;  // multiplied in the step that needs them, at whose head all loads are waited for
  const auto scales_of = [&](int block) {
    const int b = min(block, a.blocks - 1);
    next_ws = ws[b];
#pragma unroll
    for (int j = 0; j < COLS; ++j) next[j] = FROM_ROWS ? x_scales[b * held + m[j]] : a.xs[(int64_t)b * a.rows + m0 + m[j]];
  };
  scales_of(wave);
  int now = 0;
  for (int block = wave; block < a.blocks; block += WAVES) {
    float scale[COLS];
#pragma unroll
    for (int j = 0; j < COLS; ++j) scale[j] = next[j] * next_ws;
    __builtin_amdgcn_sched_barrier(0);
    scales_of(block + WAVES);
    const int last = now == 0 ? STAGES - 1 : now - 1;  // read in the step before
    __builtin_amdgcn_sched_barrier(0);
    fetch(block + (STAGES - 1) * WAVES, last);
    wait_loads<kLoads *(STAGES - 1)>();
    __builtin_amdgcn_sched_barrier(0);
    const uint8_t *const stage = mine + now * kStage;
    const auto operand = [&](int row, u32x4 (&to)[2]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) to[h] = *(const u32x4 *)(stage + row * kBlock + 16 * ((g + 4 * h) ^ (r >> 1)));
    };
    u32x4 w[2], x[COLS][2];
    operand(r, w);
#pragma unroll
    for (int j = 0; j < COLS; ++j) {
      if constexpr (FROM_ROWS) {
#pragma unroll
        for (int h = 0; h < 2; ++h) x[j][h] = *(const u32x4 *)(x_codes + (m[j] * a.blocks + block) * kBlock + 16 * (g + 4 * h));
      } else {
        operand(16 + 16 * j + r, x[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < COLS; ++j) sum[j] += block_product(w[0], w[1], x[j][0], x[j][1]) * scale[j];
    wait_loads<63>();  // the stage has been read before it is filled again
    __builtin_amdgcn_sched_barrier(0);
    now = now == STAGES - 1 ? 0 : now + 1;
  }
  __syncthreads();  // (for the loads under way too)
  f32x4 *const part = (f32x4 *)lds;  // [wave][column][lane]
  static_assert(COLS * 64 * 16 <= STAGES * kStage, "a wave's sums fit its stages");
#pragma unroll
  for (int j = 0; j < COLS; ++j) part[(wave * COLS + j) * 64 + lane] = sum[j];
  __syncthreads();
  for (int j = wave; j < COLS; j += WAVES) {
    const int row = m0 + 16 * j + r, n = n0 + 4 * g;
    f32x4 total = part[j * 64 + lane];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) total += part[(v * COLS + j) * 64 + lane];
    if (row < a.rows && n < a.outputs) store4<T>(a.y + row * a.y_stride + n, total, a.outputs - n);
  }
}

}  // namespace rnswino
