// Attention over the 4-bit cache on the matrix cores.
#pragma once
#include <type_traits>

#include "cache4.hpp"

namespace rnswino {

// s = scale q k over the positions that a row sees, p = softmax(s), o = sum p v, in one pass over the cache with the running maximum m and sum l of each row.
//
// Rows are (new token, head of the group) of one request and key head, token-major, in tiles of 16: the heads that share a key head read it once.  A wave takes 64
// positions at a time and computes S^T = K Q^T, then O^T = V^T P^T; a lane holds one row (lane % 16) in the results of both, so the statistics of a row and
// the factor that rescales its sums need nothing of other lanes but the join of its four lanes' maxima.
//
// K Q^T: v_mfma_scale_f32_16x16x128 multiplies the cache's codes and scales as they lie in memory: a lane's operand is one block of 32 dimensions of a position, 16 bytes and
// a scale byte, with no instruction in between.  At its full rate the other operand has 6 bits at most, so a query, times scale log2(e), is the sum of four pieces in e2m3 (2 bits of
// exponent, 3 of fraction), under powers of two 2^4 apart.  A piece leaves at most 1/15 of the largest magnitude of a block of 32, and 1/16 of that each further piece, so the four are
// within 2^-15.9 of it (three, 2^-11.9, showed in sharp rows).  Four such products take 64 cycles of the matrix cores for 16 positions, rows and 128 dimensions, as many as bfloat16,
// and save the conversion of the keys, 64 of a wave's 400 vector instructions a step.  The products start from -m, so that exp2 of their results are the weights.
// Key rows r of sub-tile u are the positions 16 (r / 4) + 4u + r % 4, so that lane group g = lane / 16 ends up with S of the positions 16g .. 16g + 15 in order, which are the
// contraction slots that it holds in the second product.
//
// V^T P^T: v_mfma_f32_16x16x32_bf16.  The values' scales lie along the wrong axis for the scaled instruction, so a conversion turns a byte and a scale into two bfloat16, which
// is exact (a code has two significant bits), and they go into LDS position by position and are read transposed.  P is rounded to bfloat16, 2^-8 of each weight at
// most, as far as the result's own rounding; with rows of 16-bit floats, whose 11 significant bits would show it, P is the sum of two bfloat16, with two products.  l is the sum of
// the weights before that (the sum of the rounded ones, by a product with ones, is 128 vector cycles cheaper, but its error adds to the weights' own: twice 2^-8 at worst).  Sums and
// statistics are in 32 bits.
struct AttendArgs {
  const uint16_t *q;
  uint16_t *out;
  Cache4 cache;
  const int32_t *table, *lens, *row_start;
  float *part;       // per unit and split
  int64_t q_stride, out_stride;
  int32_t requests, tokens, q_heads, group, width, window, splits, share, tiles, tile_rows;
  float factor;      // scale log2(e): scores are in powers of two
};

constexpr int kAttendWaves = 4, kAttendStep = 64;
// What a split of a tile of rows leaves: the rows' sums, then (m, l) of each.
constexpr int part_floats(int rows, int dim) { return rows * (dim + 2); }
constexpr float kNothing = -__builtin_inff();

// Two bfloat16 of codes 2n and 2n + 1 of a word.
template <int BYTE>
__device__ __forceinline__ uint32_t two_of(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
__device__ __forceinline__ bf16x8 eight_of(uint32_t codes, float scale) {
  return __builtin_bit_cast(bf16x8, u32x4{two_of<0>(codes, scale), two_of<1>(codes, scale), two_of<2>(codes, scale), two_of<3>(codes, scale)});
}

// The largest of a row's four lanes (16 apart), in all of them.
__device__ __forceinline__ float row_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// What row tile `tile` of the packed rows is: tile numbers of request i begin at floor(first row / 16) + i, which leaves every request its ceil(rows / 16).
struct TileOf {
  int request, row, rows;  // the tile's first row in the request, the request's rows
};
__device__ __forceinline__ int first_row(const AttendArgs &a, int request) {  // never outside the packed rows (the host keeps tokens * group below 2^31)
  return min(max(a.row_start[request], 0), a.tokens) * a.group;
}
template <int ROWS>
__device__ __forceinline__ TileOf tile_of(const AttendArgs &a, int tile) {
  if (a.tiles == a.requests) return {tile, 0, first_row(a, tile + 1) - first_row(a, tile)};  // one tile each
  // the last request whose first tile is `tile` or an earlier one, by 64 of them at a time, a lane each
  const int lane = threadIdx.x & 63;
  int i = 0, there = a.requests;
  while (there > 1) {
    const int step = (there + 63) / 64, at = lane * step;
    const uint64_t begun = __ballot(lane == 0 || (at < there && first_row(a, i + at) / ROWS + i + at <= tile));
    const int last = (63 - __builtin_clzll(begun)) * step;
    i += last, there = min(step, there - last);
  }
  const int first = first_row(a, i), row = (tile - first / ROWS - i) * ROWS;
  if (row < 0) return {i, 0, 0};  // in front of the first request, whose rows need not be q's first: no rows
  return {i, row, first_row(a, i + 1) - first};
}

// Whether a request with one tile has more rows than the caller promised and the tile holds.  Its results are NaN.
template <int ROWS>
__device__ __forceinline__ bool too_many(const AttendArgs &a, TileOf tile) {
  return tile.rows > ROWS && a.tiles == a.requests;
}
template <typename T, int D>
__device__ void nan_rows(const AttendArgs &a, TileOf tile, int head) {
  uint16_t *const out = a.out + (int64_t)(first_row(a, tile.request) / a.group) * a.out_stride + (int64_t)head * a.group * D;
  for (int64_t i = threadIdx.x; i < (int64_t)tile.rows * D; i += blockDim.x) {
    const int row = (int)(i / D);
    out[row / a.group * a.out_stride + row % a.group * D + i % D] = T::one(__builtin_nanf(""));
  }
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

// A tile's positions [from, to), in steps of 64 of which a workgroup takes a.share (the host's choice, so that short requests take part in few workgroups); `used` have a part.
struct Span {
  int from, to, steps, used;
};
template <int ROWS>
__device__ __forceinline__ Span span_of(const AttendArgs &a, TileOf tile, int len, int fresh) {
  const int last_token = min(tile.row + ROWS - 1, tile.rows - 1) / a.group, first_token = tile.row / a.group;
  const int to = (int)min((int64_t)max(len - fresh + last_token + 1, 0), (int64_t)a.width << a.cache.page_shift);
  const int from = a.window ? (max(len - fresh + first_token + 1 - a.window, 0) & ~15) : 0;
  const int steps = to > from ? (to - from + kAttendStep - 1) / kAttendStep : 0;
  // (a tile longer than the host was told is shared out evenly)
  const int share = max(a.share, (steps + a.splits - 1) / a.splits);
  return {from, to, steps, steps ? (steps + share - 1) / share : 1};
}
__device__ __forceinline__ int share_of(const AttendArgs &a, Span span) { return max(a.share, (span.steps + a.splits - 1) / a.splits); }

template <typename T, int D>
struct AttendTile {
  // first product: blocks of 32 dimensions, four a product (a fourth of D = 96 is zero in the query); with D = 64 two pieces of the query share one
  static constexpr int kPieces = 4;
  static constexpr int kChunks = D == 256 ? 2 : 1;  // operands of keys, 16 bytes a lane each
  static constexpr int kProducts = D == 64 ? kPieces / 2 : kPieces * kChunks;
  static constexpr int kParts = __is_same(T, F16) ? 2 : 1;  // of a weight
  // values: a lane's dimensions of a position, words of codes, and scales that they lie under
  static constexpr int kDims = D / 4, kWords = D / 32, kBlocks = D == 96 || D == 256 ? 2 : 1;
  // Bytes of a position's values in LDS: with 32 more than 2D, the 32 bytes that a transposed read takes of each of four positions lie in different banks; and with 128 more between the positions
  // of different lane groups (16, or 8 where half a step is kept), the other half of the banks is the next group's: 2 cycles a read instead of 4.
  static constexpr int kRow = 2 * D + 32, kGroup = 128, kSlab = kAttendStep * kRow + 4 * kGroup;

  static __device__ __forceinline__ int key_block(int chunk, int g) { return D == 64 ? g & 1 : D == 96 ? min(g, 2) : 4 * chunk + g; }
  // block of a lane's dimensions [8s, 8s + 8), relative to its first
  static __device__ __forceinline__ int first_block(int g) { return min(g * kDims / 32, D / 32 - kBlocks); }
  static __device__ __forceinline__ int block_of(int g, int s) { return (g * kDims + 8 * s) / 32 - first_block(g); }

  // A row's query as operands of the products: lane (r, g) holds block key_block(chunk, g), a piece after another.
  struct Query {
    u32x6 codes[kProducts];
    int scale[kChunks];  // byte p: of piece p (D = 64: of piece 2p + g / 2)
  };
};

// A query's words as they lie in memory; zeros where there is no row.
template <typename T, int D>
struct RawQuery {
  u32x4 words[AttendTile<T, D>::kChunks][4];
  __device__ __forceinline__ void load(const AttendArgs &a, int64_t token, int head, int g, bool live) {
    using X = AttendTile<T, D>;
    const uint16_t *from = a.q + token * a.q_stride + (int64_t)head * D;
#pragma unroll
    for (int c = 0; c < X::kChunks; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        words[c][i] = *(const u32x4 *)(from + 32 * X::key_block(c, g) + 8 * i);
        if (!live || (D == 96 && g == 3)) words[c][i] = u32x4{0, 0, 0, 0};
      }
  }
};

template <typename T, int D>
__device__ __forceinline__ void make_query(const AttendArgs &a, const RawQuery<T, D> &raw, int g, typename AttendTile<T, D>::Query &query) {
  using X = AttendTile<T, D>;
#pragma unroll
  for (int c = 0; c < X::kChunks; ++c) {
    // even and odd dimensions: the conversion takes them in turn
    f32x16 even, odd;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        even[4 * i + e] = T::low(raw.words[c][i][e]) * a.factor;
        odd[4 * i + e] = T::high(raw.words[c][i][e]) * a.factor;
        most = max(most, max(__float_as_uint(even[4 * i + e]) & 0x7FFFFFFFu, __float_as_uint(odd[4 * i + e]) & 0x7FFFFFFFu));
      }
    }
    // the smallest power of two (of at least 2^-110) under which the block's largest magnitude is at most 7.5 = 1.875 2^2; a block with an infinity or a NaN gets the scale NaN
    const int byte = max((int)(most >> 23) - 2 + ((most & 0x7FFFFFu) > 0x700000u ? 1 : 0), 17);
    u32x6 piece[X::kPieces];
#pragma unroll
    for (int p = 0; p < X::kPieces; ++p) {
      const float scale = __uint_as_float((uint32_t)(byte - 4 * p) << 23);
      piece[p] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, scale);
      const f32x32 taken = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(piece[p], scale);
#pragma unroll
      for (int i = 0; i < 16; ++i) even[i] -= taken[2 * i], odd[i] -= taken[2 * i + 1];
      // The conversion writes its first results before it has read its last operands: these are still needed behind it (here for what the piece leaves), so that they do not share registers.
      asm volatile("" ::"v"(even), "v"(odd));
    }
    const bool broken = most >= 0x7F800000u;
    if constexpr (D == 64) {
#pragma unroll
      for (int i = 0; i < X::kProducts; ++i) query.codes[i] = g < 2 ? piece[2 * i] : piece[2 * i + 1];
      const int first = byte - 4 * (g >> 1);
      query.scale[c] = broken ? -1 : first | (first - 8) << 8;
    } else {
#pragma unroll
      for (int p = 0; p < X::kPieces; ++p) query.codes[p * X::kChunks + c] = piece[p];
      query.scale[c] = broken ? -1 : byte | (byte - 4) << 8 | (byte - 8) << 16 | (byte - 12) << 24;
    }
  }
}

// 16 positions' keys by 16 queries, added to `s`.
template <typename T, int D, int PRODUCT = 0>
__device__ __forceinline__ f32x4 scores(const u32x4 (&key)[AttendTile<T, D>::kChunks], const uint32_t (&scale)[AttendTile<T, D>::kChunks], int shift,
                                        const typename AttendTile<T, D>::Query &query, f32x4 s) {
  using X = AttendTile<T, D>;
  if constexpr (PRODUCT < X::kProducts) {
    constexpr int c = PRODUCT % X::kChunks, byte = PRODUCT / X::kChunks;
    const i32x8 k = {(int)key[c].x, (int)key[c].y, (int)key[c].z, (int)key[c].w, 0, 0, 0, 0};
    const u32x6 q = query.codes[PRODUCT];
    const i32x8 qq = {(int)q[0], (int)q[1], (int)q[2], (int)q[3], (int)q[4], (int)q[5], 0, 0};
    s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, qq, s, 4, 2, 0, (int)(scale[c] >> shift), byte, query.scale[c]);
    return scores<T, D, PRODUCT + 1>(key, scale, shift, query, s);
  } else {
    return s;
  }
}

// Where a lane finds a position's scale bytes from `block` on: in which word behind the scales of the position's 16 (PAIR, for two bytes of D = 96, whose threes lie across words: in which
// two words), and how far up.  They are loaded as words: a byte's load would be widened, and so waited for, where the compiler likes, which was before the step that asks for it ends (8 prompts of 2048 behind 2048,
// 8 and 4 heads of 256: 1005 us so, 656 with words).
template <int D, bool PAIR = false>
struct ScalesAt {
  static constexpr bool kTwo = PAIR && D == 96;
  typedef uint32_t u32x2_4 __attribute__((ext_vector_type(2), aligned(4)));
  typedef std::conditional_t<kTwo, u32x2_4, uint32_t> Word;
  int word, shift;
  __device__ __forceinline__ ScalesAt(int position, int block) {
    const int four = (position & ~3) * (D / 32), at = (position & 3) * (D / 32) + block, in_four = kTwo ? min(at & ~3, 4) : at & ~3;
    word = four + in_four, shift = 8 * (at - in_four);
  }
  __device__ __forceinline__ uint32_t byte(Word w, int more) const {
    if constexpr (kTwo) return (uint32_t)(__builtin_bit_cast(uint64_t, w) >> shift) >> 8 * more & 255;
    else return w >> shift >> 8 * more & 255;
  }
};

// A row's running maximum: weights are taken relative to it, and it is only moved where a step's largest score exceeds it by more than 2^kGrowth in weight; until then weights are
// at most that, as exact as before in floating point.
constexpr float kGrowth = 8.0f;
struct Level {
  float minus = 0;    // -m, in log2; what the products start from
  bool unset = true;  // nothing seen yet
  __device__ __forceinline__ f32x4 start() const { return f32x4{minus, minus, minus, minus}; }
  __device__ __forceinline__ bool grows(float top) const { return top > (unset ? kNothing : kGrowth); }
  // Moves m by `shift` to the step's largest score; returns the factor of the sums so far.
  __device__ __forceinline__ float move(float top, float &shift) {
    shift = unset ? (top == kNothing ? 0.0f : top) : fmaxf(top, 0.0f);
    const float keep = unset ? 1.0f : __builtin_amdgcn_exp2f(-shift);
    unset = unset && top == kNothing;
    minus -= shift;
    return keep;
  }
  __device__ __forceinline__ float m() const { return unset ? kNothing : -minus; }
};

template <int WORDS>
__device__ __forceinline__ void load_words(const uint8_t *from, uint32_t (&w)[WORDS]) {
  if constexpr (WORDS == 2) {
    const u32x2 v = *(const u32x2 *)from;
    w[0] = v.x, w[1] = v.y;
  } else if constexpr (WORDS % 4 == 0) {
#pragma unroll
    for (int i = 0; i < WORDS / 4; ++i) {
      const u32x4 v = *(const u32x4 *)(from + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * i + e] = v[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = *(const uint32_t *)(from + 4 * i);
  }
}

// Values of eight positions from `position`, transposed: lane r of its group gets dimension dim + r of all eight.  (The instruction: lane i of 16 gives the place of four
// dimensions of position i / 4 of four, and gets dimension i of the four positions.)
template <int ROW>
__device__ __forceinline__ bf16x8 values_of(const uint8_t *slab, int position, int dim, int r) {  // slab: the lane group's
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 *lds4;
  const uint8_t *at = slab + (position + (r >> 2)) * ROW + (dim + 4 * (r & 3)) * 2;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 4 * ROW));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Few rows: the waves of a workgroup take the 64 positions in turn, each with its own statistics, and join at the end; where the tile has several workgroups they
// leave their sums to k_cache4_join.  Bound by memory: a wave's next keys and values are asked for as soon as the registers of the present ones are free, and values go through LDS 32
// positions at a time, so that three workgroups fit a compute unit.  (Of all instances one has not the registers for that: bfloat16 rows with heads of 96 keep two in scratch, 12 bytes a lane.)
template <typename T, int D>
__global__ __launch_bounds__(64 * kAttendWaves, D == 256 ? 2 : 3) void k_cache4_attend(AttendArgs a) {
  using X = AttendTile<T, D>;
  constexpr int kSlab = 32 * X::kRow + 4 * X::kGroup;
  __shared__ __align__(16) uint8_t lds[kAttendWaves * kSlab + kAttendWaves * 16 * 8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  // (units first: the parts of a short request's tile that have nothing to do would all be on the same XCDs, 110 -> 177 us with 16 parts for 64 requests of 500 to 16000 positions)
  const int units = a.tiles * a.cache.heads, split = blockIdx.x / units, unit = blockIdx.x - split * units;
  const int head = unit % a.cache.heads, tile_id = unit / a.cache.heads;
  const TileOf tile = tile_of<16>(a, tile_id);
  const int len = a.lens[tile.request];
  if (tile.row >= tile.rows) return;
  if (too_many<16>(a, tile)) {
    if (split == 0) nan_rows<T, D>(a, tile, head);
    return;
  }
  const int fresh = tile.rows / a.group;
  const int first_token = first_row(a, tile.request) / a.group;
  const int32_t *pages = a.table + (int64_t)tile.request * a.width;
  const Span span = span_of<16>(a, tile, len, fresh);
  if (split >= span.used) return;
  const int share = share_of(a, span), step_to = min((split + 1) * share, span.steps);

  // this lane's 16 positions of a step, as rows of the first product: their page (behind the span: that of its last), and their first row in the cache (without a page: the cache's first)
  const auto page_at = [&](int step) { return pages[min(span.from + step * kAttendStep + 16 * (r >> 2), span.to - 1) >> a.cache.page_shift]; };
  const auto row_of = [&](int step, int page) {
    const uint32_t of = (uint32_t)page < (uint32_t)a.cache.pages ? (uint32_t)page : 0u;
    const uint32_t in_page = (uint32_t)(span.from + step * kAttendStep + 16 * (r >> 2)) & ((1u << a.cache.page_shift) - 1);
    return ((of * (uint32_t)a.cache.heads + head) << a.cache.page_shift) + in_page;  // the host keeps the rows below 2^32
  };
  u32x4 key[4][X::kChunks];
  uint32_t vw[4][X::kWords], ks[4][X::kChunks];
  typename ScalesAt<D, true>::Word vs[4];
  // a lane's places in a step's 64 positions, of which sub-tile u is 4u rows on
  const ScalesAt<D> k_scales(r & 3, X::key_block(0, g));
  const ScalesAt<D, true> v_scales(r & 3, X::first_block(g));
  const uint8_t *const k_lane = a.cache.k + (r & 3) * (D / 2) + 16 * X::key_block(0, g), *const ks_lane = a.cache.k_scale + k_scales.word;
  const uint8_t *const v_lane = a.cache.v + (r & 3) * (D / 2) + g * (X::kDims / 2), *const vs_lane = a.cache.v_scale + v_scales.word;
  const auto load_keys = [&](uint32_t row) {
    const uint8_t *const codes = k_lane + (uint64_t)row * (D / 2), *const scales = ks_lane + (uint64_t)row * (D / 32);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int c = 0; c < X::kChunks; ++c) {
        key[u][c] = *(const u32x4 *)(codes + 4 * u * (D / 2) + 64 * c);
        ks[u][c] = *(const uint32_t *)(scales + 4 * u * (D / 32) + 4 * c);
      }
  };
  const auto load_values = [&](uint32_t row) {
    const uint8_t *const codes = v_lane + (uint64_t)row * (D / 2), *const scales = vs_lane + (uint64_t)row * (D / 32);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      load_words<X::kWords>(codes + 4 * u * (D / 2), vw[u]);
      vs[u] = *(const typename ScalesAt<D, true>::Word *)(scales + 4 * u * (D / 32));
    }
  };
  // this lane's row: its query, asked for before keys and values so that it is made ready while they arrive, and the positions it sees (no row: the last one's)
  const int row = min(tile.row + r, tile.rows - 1), row_token = row / a.group;
  const bool live = tile.row + r < tile.rows;
  RawQuery<T, D> raw;
  raw.load(a, first_token + row_token, head * a.group + row % a.group, g, live);
  int step = split * share + wave, page0 = -1, page1 = -1;
  uint32_t at = 0;
  if (step < step_to) {
    page0 = page_at(step), page1 = page_at(step + kAttendWaves);
    at = row_of(step, page0);
    load_keys(at);
  }
  const int position = len - fresh + row_token;
  const int seen_to = min(min(position + 1, len), span.to);
  const int seen_from = a.window ? max(position + 1 - a.window, 0) : 0;
  // positions that all rows of the tile see
  const int common_to = min(min(len - fresh + tile.row / a.group + 1, len), span.to);
  const int common_from = a.window ? max(len - fresh + min(tile.row + 15, tile.rows - 1) / a.group + 1 - a.window, 0) : 0;
  typename X::Query query;
  make_query<T, D>(a, raw, g, query);
  if (step < step_to) load_values(at);

  f32x4 sum[D / 16];
#pragma unroll
  for (int d = 0; d < D / 16; ++d) sum[d] = f32x4{0, 0, 0, 0};
  Level level;
  float l = 0;  // of the lane's positions
  uint8_t *const slab = lds + wave * kSlab;

  for (; step < step_to; step += kAttendWaves) {
    const int base = span.from + step * kAttendStep;
    const bool there = (uint32_t)page0 < (uint32_t)a.cache.pages && base + 16 * (r >> 2) < span.to;
    const bool mine_there = __shfl((int)there, 4 * g) != 0;  // of this lane's positions of the second product
    const int page2 = page_at(step + 2 * kAttendWaves);
    f32x4 s[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] = scores<T, D>(key[u], ks[u], k_scales.shift, query, level.start());
    const uint32_t next = row_of(step + kAttendWaves, page1);  // behind the last step: a row of the cache that nothing is made of
    load_keys(next);
    // values of sub-tiles u and u + 1 into the slab; a position's scales may be anything where there is none, its codes are finite whatever they are; a NaN scale is kept out of
    // the product, where it would reach rows that do not see it, and makes the scores of those that do NaN
    uint32_t bad = 0;
    const auto put_values = [&](int first) {
#pragma unroll
      for (int u = first; u < first + 2; ++u) {
        const bool real = there && base + 16 * (r >> 2) + 4 * u + (r & 3) < span.to;
#pragma unroll
        for (int w = 0; w < X::kWords; ++w) {
          uint32_t byte = v_scales.byte(vs[u], 0);
          if (X::kBlocks == 2 && X::block_of(g, w)) byte = v_scales.byte(vs[u], 1);
          if (byte == 255 || !real) byte = 1;
          *(bf16x8 *)(slab + (8 * (r >> 2) + 4 * (u & 1) + (r & 3)) * X::kRow + (r >> 2) * X::kGroup + (g * X::kDims + 8 * w) * 2) = eight_of(vw[u][w], __uint_as_float(byte << 23));
        }
      }
    };
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      bool broken = v_scales.byte(vs[u], 0) == 255;
      if constexpr (X::kBlocks == 2) broken |= v_scales.byte(vs[u], 1) == 255;
      if (broken && there && base + 16 * (r >> 2) + 4 * u + (r & 3) < span.to) bad |= 1u << u;
    }
    put_values(0);
    // Steps that all rows see whole are not masked with heads of 64 (22 requests of 1393 positions, 6 and 2 heads: 11.4 us, 10.5 so; with others the branch costs registers that they have not)
    if (D != 64 || !(base >= common_from && base + kAttendStep <= common_to && __all(there))) {
      const uint32_t first = base + 16 * g - seen_from, seen = mine_there && seen_to > seen_from ? seen_to - seen_from : 0;
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[u][i] = first + 4 * u + i < seen ? s[u][i] : kNothing;
    }
    float top = kNothing;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[u][i]);
    if (__any(bad != 0)) {
      bad |= __shfl_xor((int)bad, 16);
      bad |= __shfl_xor((int)bad, 32);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t of = (uint32_t)__shfl((int)bad, 4 * g + i);  // bit u: position 16g + 4u + i
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if ((of >> u & 1) && s[u][i] != kNothing) s[u][i] = __builtin_nanf("");
      }
    }
    top = row_max(top);
    if (__any(level.grows(top))) {
      float shift;
      const float keep = level.move(top, shift);
      l *= keep;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) sum[d] *= keep;
#pragma unroll
      for (int u = 0; u < 4; ++u) s[u] -= shift;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 weight[X::kParts];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(s[2 * h + e / 4][e % 4]);
        l += p;
        weight[0][e] = (__bf16)p;
        if constexpr (X::kParts == 2) weight[1][e] = (__bf16)(p - (float)weight[0][e]);
      }
      if (h == 1) {
        put_values(2);
        load_values(next);
      }
      // the wave's own values, written by its other lanes
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      constexpr int kTogether = 4;  // reads in flight
#pragma unroll
      for (int d = 0; d < D / 16; d += kTogether) {
        bf16x8 value[kTogether];
#pragma unroll
        for (int e = 0; e < kTogether; ++e)
          if (d + e < D / 16) value[e] = values_of<X::kRow>(slab + g * X::kGroup, 8 * g, 16 * (d + e), r);
#pragma unroll
        for (int e = 0; e < kTogether; ++e)
#pragma unroll
          for (int part = 0; part < X::kParts; ++part)
            if (d + e < D / 16) sum[d + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value[e], weight[part], sum[d + e], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    page0 = page1, page1 = page2;
  }
  l = row_sum(l);

  // join the waves: each leaves its sums in its slab ([row][D] in 32 bits), then m and l behind all slabs
  float *mine = (float *)slab, *stats = (float *)(lds + kAttendWaves * kSlab);
  if (g == 0) {
    stats[(wave * 16 + r) * 2] = level.m();
    stats[(wave * 16 + r) * 2 + 1] = l;
  }
#pragma unroll
  for (int d = 0; d < D / 16; ++d) *(f32x4 *)(mine + r * D + 16 * d + 4 * g) = sum[d];
  __syncthreads();
  for (int at = threadIdx.x * 4; at < 16 * D; at += 64 * kAttendWaves * 4) {
    const int row_at = at / D;
    if (tile.row + row_at >= tile.rows) break;
    float best = kNothing;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) best = fmaxf(best, stats[(w * 16 + row_at) * 2]);
    const float used = best == kNothing ? 0.0f : best;
    f32x4 joined = {0, 0, 0, 0};
    float all = 0;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(stats[(w * 16 + row_at) * 2] - used);
      joined += *(const f32x4 *)((const float *)(lds + w * kSlab) + at) * f;
      all += stats[(w * 16 + row_at) * 2 + 1] * f;
    }
    if (span.used > 1) {
      float *to = a.part + ((int64_t)unit * a.splits + split) * part_floats(16, D);
      *(f32x4 *)(to + at) = joined;
      if (at % D == 0) {
        to[16 * D + 2 * row_at] = best;
        to[16 * D + 2 * row_at + 1] = all;
      }
    } else {
      const float inverse = all > 0 || all != all ? 1.0f / all : 0.0f;  // a row that sees nothing is 0
      const int rr = tile.row + row_at;
      uint16_t *to = a.out + (first_token + rr / a.group) * a.out_stride + (int64_t)(head * a.group + rr % a.group) * D + at % D;
      *(u32x2 *)to = u32x2{T::pair(joined[0] * inverse, joined[1] * inverse), T::pair(joined[2] * inverse, joined[3] * inverse)};
    }
  }
}

// Many rows: a workgroup's four waves hold TILES x 16 rows each and take the same 64 positions.  Keys come straight from memory to every wave.  Values are converted once, a quarter by each wave, into one of two
// stages in LDS.

template <typename T, int D, int TILES>
__global__ __launch_bounds__(256, 2) void k_cache4_attend_many(AttendArgs a) {
  using X = AttendTile<T, D>;
  constexpr int kRows = 64 * TILES;
  __shared__ __align__(16) uint8_t lds[2][X::kSlab];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int units = a.tiles * a.cache.heads, split = blockIdx.x / units, unit = blockIdx.x - split * units;
  const int head = unit % a.cache.heads;
  // the last rows see most: they are begun first
  const TileOf tile = tile_of<kRows>(a, a.tiles - 1 - unit / a.cache.heads);
  if (tile.row >= tile.rows) return;
  if (too_many<kRows>(a, tile)) {
    if (split == 0) nan_rows<T, D>(a, tile, head);
    return;
  }
  const int fresh = tile.rows / a.group;
  const int64_t first_token = first_row(a, tile.request) / a.group;
  const int len = a.lens[tile.request];
  const int32_t *pages = a.table + (int64_t)tile.request * a.width;
  const Span span = span_of<kRows>(a, tile, len, fresh);
  if (split >= span.used) return;

  typename X::Query query[TILES];
  int seen_to[TILES], seen_from[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const bool live = tile.row + (wave * TILES + t) * 16 + r < tile.rows;
    const int row = min(tile.row + (wave * TILES + t) * 16 + r, tile.rows - 1), row_token = row / a.group;
    const int position = len - fresh + row_token;
    seen_to[t] = min(min(position + 1, len), span.to);
    seen_from[t] = a.window ? max(position + 1 - a.window, 0) : 0;
    RawQuery<T, D> raw;
    raw.load(a, first_token + row_token, head * a.group + row % a.group, g, live);
    make_query<T, D>(a, raw, g, query[t]);
  }
  const int last_token = min(tile.row + kRows - 1, tile.rows - 1) / a.group, first_of_tile = tile.row / a.group;
  const int tile_from = span.from, tile_to = span.to;
  // positions that all rows of the tile see
  const int common_to = min(min(len - fresh + first_of_tile + 1, len), span.to);
  const int common_from = a.window ? max(len - fresh + last_token + 1 - a.window, 0) : 0;
  const int share = share_of(a, span), step_from = split * share, step_to = min(step_from + share, span.steps);

  f32x4 sum[TILES][D / 16];
  float l[TILES];  // of the lane's positions
  Level level[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    l[t] = 0;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) sum[t][d] = f32x4{0, 0, 0, 0};
  }

  const int place = 4 * wave + (r & 3);  // of this wave's values among a page's 16: the positions 16 (r / 4) + place
  // The page of this lane's 16 positions of a step (behind the tile's last: the last one's), and their first row in the cache (without a page: the cache's first). No branches: one
  // would part the step's products from what runs beside them.
  const auto page_at = [&](int step) { return pages[min(tile_from + step * kAttendStep + 16 * (r >> 2), tile_to - 1) >> a.cache.page_shift]; };
  const auto there_at = [&](int step, int page) { return (uint32_t)page < (uint32_t)a.cache.pages && tile_from + step * kAttendStep + 16 * (r >> 2) < tile_to; };
  const auto row_of = [&](int step, int page) {
    const uint32_t of = (uint32_t)page < (uint32_t)a.cache.pages ? (uint32_t)page : 0u;
    const uint32_t in_page = (uint32_t)(tile_from + step * kAttendStep + 16 * (r >> 2)) & ((1u << a.cache.page_shift) - 1);
    return ((of * (uint32_t)a.cache.heads + head) << a.cache.page_shift) + in_page;  // the host keeps the rows below 2^32
  };
  struct Keys {
    u32x4 codes[4][X::kChunks];
    uint32_t scale[4][X::kChunks];
  };
  uint32_t vw[X::kWords];
  typename ScalesAt<D, true>::Word vs;
  Keys key;
  // a lane's places in a step's 64 positions, of which sub-tile u is 4u rows on
  const ScalesAt<D> k_scales(r & 3, X::key_block(0, g));
  const ScalesAt<D, true> v_scales(place, X::first_block(g));
  const uint8_t *const k_lane = a.cache.k + (r & 3) * (D / 2) + 16 * X::key_block(0, g), *const ks_lane = a.cache.k_scale + k_scales.word;
  const uint8_t *const v_lane = a.cache.v + place * (D / 2) + g * (X::kDims / 2), *const vs_lane = a.cache.v_scale + v_scales.word;
  const auto load_keys = [&](uint32_t row) {
    const uint8_t *const codes = k_lane + (uint64_t)row * (D / 2), *const scales = ks_lane + (uint64_t)row * (D / 32);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int c = 0; c < X::kChunks; ++c) {
        key.codes[u][c] = *(const u32x4 *)(codes + 4 * u * (D / 2) + 64 * c);
        key.scale[u][c] = *(const uint32_t *)(scales + 4 * u * (D / 32) + 4 * c);
      }
  };
  const auto load_values = [&](uint32_t row) {
    load_words<X::kWords>(v_lane + (uint64_t)row * (D / 2), vw);
    vs = *(const typename ScalesAt<D, true>::Word *)(vs_lane + (uint64_t)row * (D / 32));
  };
  // into stage `to`; positions without a page, or behind the tile's last, get a scale of next to nothing.  Returns whether one is NaN
  __shared__ uint32_t broken[2][4];
  const auto put_values = [&](int step, int page, int to) {
    const bool real = there_at(step, page) && tile_from + step * kAttendStep + 16 * (r >> 2) + place < tile_to;
    bool bad = false;
#pragma unroll
    for (int w = 0; w < X::kWords; ++w) {
      uint32_t byte = v_scales.byte(vs, 0);
      if (X::kBlocks == 2 && X::block_of(g, w)) byte = v_scales.byte(vs, 1);
      bad |= byte == 255 && real;
      if (byte == 255 || !real) byte = 1;
      *(bf16x8 *)(lds[to] + (16 * (r >> 2) + place) * X::kRow + (r >> 2) * X::kGroup + (g * X::kDims + 8 * w) * 2) = eight_of(vw[w], __uint_as_float(byte << 23));
    }
    // bit r: the wave's position of row r holds a NaN block
    const uint64_t any = __ballot(bad);
    broken[to][wave] = (uint32_t)((any | any >> 16 | any >> 32 | any >> 48) & 0xFFFF);  // by all lanes: a branch would cut the step in two
  };

  // pages of this step and the next two (a page is asked for a step before its rows are), and the next step's rows
  int page0 = 0, page1 = 0, page2 = 0;
  uint32_t row1 = 0;
  const auto take = [&](bool masked, int step, int now, bool mine_there) {
    const int base = tile_from + step * kAttendStep;
    const int page3 = page_at(step + 3);
    f32x4 s[TILES][4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int t = 0; t < TILES; ++t) s[t][u] = scores<T, D>(key.codes[u], key.scale[u], k_scales.shift, query[t], level[t].start());
    // the next keys go into the registers that the products have read (asked for earlier they would need others, and copies that wait for them), and the products run while the
    // next values are converted; behind the last step the addresses are those of the cache's first rows
    __builtin_amdgcn_sched_barrier(0);
    load_keys(row1);
    put_values(step + 1, page1, now ^ 1);
    row1 = row_of(step + 2, page2);
    load_values(row1);
    __builtin_amdgcn_sched_barrier(0);
    if (masked) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t of = broken[now][u] >> (4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = base + 16 * g + 4 * u + i;
#pragma unroll
          for (int t = 0; t < TILES; ++t) {
            if (of >> i & 1) s[t][u][i] = __builtin_nanf("");
            s[t][u][i] = mine_there && at >= seen_from[t] && at < seen_to[t] ? s[t][u][i] : kNothing;
          }
        }
      }
    }
    float top[TILES];
    bool grows = false;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      top[t] = s[t][0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top[t] = fmaxf(top[t], s[t][e / 4][e % 4]);
      top[t] = row_max(top[t]);
      grows |= level[t].grows(top[t]);
    }
    if (__any(grows)) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        float shift;
        const float keep = level[t].move(top[t], shift);
        l[t] *= keep;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) sum[t][d] *= keep;
#pragma unroll
        for (int u = 0; u < 4; ++u) s[t][u] -= shift;
      }
    }
    // half of the weights, then its products beside the other half
    bf16x8 weight[2][TILES][X::kParts];
    const auto weigh = [&](int h, int t, int e) {
      const float p = __builtin_amdgcn_exp2f(s[t][2 * h + e / 4][e % 4]);
      l[t] += p;
      weight[h][t][0][e] = (__bf16)p;
      if constexpr (X::kParts == 2) weight[h][t][1][e] = (__bf16)(p - (float)weight[h][t][0][e]);
    };
    const auto join = [&](int h, int d) {
      const bf16x8 value = values_of<X::kRow>(lds[now] + g * X::kGroup, 16 * g + 8 * h, 16 * d, r);
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int part = 0; part < X::kParts; ++part) sum[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value, weight[h][t][part], sum[t][d], 0, 0, 0);
    };
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) weigh(0, t, e);
#pragma unroll
    for (int d = 0; d < D / 16; ++d) join(0, d);
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) weigh(1, t, e);
#pragma unroll
    for (int d = 0; d < D / 16; ++d) join(1, d);
    page0 = page1, page1 = page2, page2 = page3;
  };
  const auto next_step = [&](int step, int now) {
    lds_barrier();  // stage `now` is whole, the other is free
    const int base = tile_from + step * kAttendStep;
    const bool there = there_at(step, page0);
    const uint32_t bad = broken[now][0] | broken[now][1] | broken[now][2] | broken[now][3];
    const bool whole = base >= common_from && base + kAttendStep <= common_to && __all(there) && __builtin_amdgcn_readfirstlane(bad) == 0;
    take(!whole, step, now, __shfl((int)there, 4 * g) != 0);
  };
  if (step_from < step_to) {
    page0 = page_at(step_from), page1 = page_at(step_from + 1), page2 = page_at(step_from + 2);
    row1 = row_of(step_from, page0);
    load_values(row1);
    load_keys(row1);
    put_values(step_from, page0, 0);
    row1 = row_of(step_from + 1, page1);
    load_values(row1);
    for (int step = step_from; step < step_to; ++step) next_step(step, (step - step_from) & 1);
  }
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const float all = row_sum(l[t]);
    const int row_at = (wave * TILES + t) * 16 + r, row = tile.row + row_at;
    if (row >= tile.rows) continue;
    if (span.used > 1) {
      float *to = a.part + ((int64_t)((a.tiles - 1 - unit / a.cache.heads) * a.cache.heads + head) * a.splits + split) * part_floats(kRows, D);
#pragma unroll
      for (int d = 0; d < D / 16; ++d) *(f32x4 *)(to + row_at * D + 16 * d + 4 * g) = sum[t][d];
      if (g == 0) {
        to[kRows * D + 2 * row_at] = level[t].m();
        to[kRows * D + 2 * row_at + 1] = all;
      }
    } else {
      const float inverse = all > 0 || all != all ? 1.0f / all : 0.0f;
      uint16_t *to = a.out + (first_token + row / a.group) * a.out_stride + (int64_t)(head * a.group + row % a.group) * D + 4 * g;
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
        *(u32x2 *)(to + 16 * d) = u32x2{T::pair(sum[t][d][0] * inverse, sum[t][d][1] * inverse), T::pair(sum[t][d][2] * inverse, sum[t][d][3] * inverse)};
    }
  }
}

// Joins the workgroups of a tile of ROWS rows, in their order: a wave a row, a lane the statistics of one workgroup (there are 64 at most), then D / 64 dimensions.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(256) void k_cache4_join(AttendArgs a) {
  constexpr int kPart = part_floats(ROWS, D), kEach = D == 64 ? 1 : D == 256 ? 4 : 2, kTogether = 8;
  typedef float each __attribute__((ext_vector_type(kEach)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int unit = blockIdx.x, head = unit % a.cache.heads;
  const TileOf tile = tile_of<ROWS>(a, unit / a.cache.heads);
  const int row_at = blockIdx.y * 4 + wave, row = tile.row + row_at;
  if (row >= tile.rows || too_many<ROWS>(a, tile)) return;
  const Span span = span_of<ROWS>(a, tile, a.lens[tile.request], tile.rows / a.group);
  if (span.used < 2) return;
  const float *from = a.part + (int64_t)unit * a.splits * kPart;
  const f32x2 stats = lane < span.used ? *(const f32x2 *)(from + (int64_t)lane * kPart + ROWS * D + 2 * row_at) : f32x2{kNothing, 0};
  float best = stats.x, all;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) best = fmaxf(best, __shfl_xor(best, d));
  const float f = __builtin_amdgcn_exp2f(stats.x - (best == kNothing ? 0.0f : best));
  all = stats.y * f;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d);
  if (lane * kEach >= D) return;
  from += row_at * D + lane * kEach;
  each total = {};
  for (int s = 0; s < span.used; s += kTogether) {
    each part[kTogether];
#pragma unroll
    for (int e = 0; e < kTogether; ++e) part[e] = *(const each *)(from + (int64_t)min(s + e, span.used - 1) * kPart);
#pragma unroll
    for (int e = 0; e < kTogether; ++e)
      if (s + e < span.used) total += part[e] * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s + e));
  }
  const float inverse = all > 0 || all != all ? 1.0f / all : 0.0f;
  uint16_t *to = a.out + ((int64_t)(first_row(a, tile.request) + row) / a.group) * a.out_stride + (int64_t)(head * a.group + row % a.group) * D + lane * kEach;
  if constexpr (kEach == 1) *to = T::one(total[0] * inverse);
  else if constexpr (kEach == 2) *(uint32_t *)to = T::pair(total[0] * inverse, total[1] * inverse);
  else *(u32x2 *)to = u32x2{T::pair(total[0] * inverse, total[1] * inverse), T::pair(total[2] * inverse, total[3] * inverse)};
}

}  // namespace rnswino
