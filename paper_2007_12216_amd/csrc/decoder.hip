// Host entry points of the decoder operators: argument checks and launches.  Nothing here allocates, synchronises or throws.
#include "rnswino.h"

#include "k_block_tables.hpp"
#include "k_cache4_attention.hpp"
#include "k_fp8.hpp"
#include "k_qk_rope.hpp"

namespace {

using namespace rnswino;

int launch_result() { return hipGetLastError() == hipSuccess ? RNSWINO_OK : RNSWINO_E_HIP; }

int log2_of(int32_t page_size) {  // of a power of two
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}
bool page_size_ok(int32_t p) { return p >= 16 && p <= 4096 && (p & (p - 1)) == 0; }
bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// A launch has fewer than 2^32 threads, in whole workgroups.
constexpr int64_t kMostThreads = (1LL << 32) - 256;

struct Range {
  const void *begin;
  int64_t bytes;
};
bool overlap(Range a, Range b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.begin), y = reinterpret_cast<uintptr_t>(b.begin);
  return x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes && a.bytes && b.bytes;
}

bool type_ok(int32_t type) { return type == RNSWINO_TYPE_BF16 || type == RNSWINO_TYPE_F16; }

// What a cache's description has to be for any call; `out` gets the kernels' form of it.
int cache_of(const rnswino_cache4_t *c, Cache4 &out) {
  if (!c || !c->k || !c->k_scale || !c->v || !c->v_scale || c->n_pages <= 0 || c->kv_heads <= 0 || c->head_dim <= 0) return RNSWINO_E_INVALID;
  if (!aligned(c->k, 16) || !aligned(c->k_scale, 16) || !aligned(c->v, 16) || !aligned(c->v_scale, 16)) return RNSWINO_E_INVALID;
  if (!page_size_ok(c->page_size) || c->head_dim % 32 || c->head_dim > 256) return RNSWINO_E_UNSUPPORTED;
  out = {(uint8_t *)c->k, (uint8_t *)c->k_scale, (uint8_t *)c->v, (uint8_t *)c->v_scale, c->n_pages, log2_of(c->page_size), c->kv_heads, c->head_dim};
  return RNSWINO_OK;
}

bool rows_ok(const void *p, int64_t stride, int64_t width) { return p && aligned(p, 16) && stride >= width && stride % 8 == 0; }

int rope_lanes(int dim) { return dim <= 64 ? 8 : dim <= 128 ? 16 : 32; }  // of a head

template <typename T, int LANES, bool TO_CACHE>
void launch_rope(const RopeArgs &a, hipStream_t stream) {
  const int64_t items = (int64_t)a.tokens * (a.q_heads + a.kv_heads * (TO_CACHE ? 2 : 1)), bytes = 2LL * a.tokens * a.dim * (a.q_heads + (TO_CACHE ? 0 : a.kv_heads));
  const dim3 grid((unsigned)((items * LANES + 255) / 256));
  // Results past the caches from what the L2s hold on (40 heads of 128: 8192 tokens 44.7 -> 35.6 us, 6400 29; smaller ones are likely to be read from there by what comes next).
  if (bytes >= (32 << 20)) hipLaunchKernelGGL((k_qk_rope<T, LANES, TO_CACHE, true>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((k_qk_rope<T, LANES, TO_CACHE, false>), grid, dim3(256), 0, stream, a);
}
template <typename T, bool TO_CACHE>
void launch_rope(const RopeArgs &a, hipStream_t stream) {
  switch (rope_lanes(a.dim)) {
    case 8: return launch_rope<T, 8, TO_CACHE>(a, stream);
    case 16: return launch_rope<T, 16, TO_CACHE>(a, stream);
    default: return launch_rope<T, 32, TO_CACHE>(a, stream);
  }
}

int rope(const rnswino_rope_t *d, const void *q, const void *k, const void *v, const void *wq, const void *wk, const float *angles, const int32_t *positions,
         const int64_t *slots, void *q_out, void *k_out, const rnswino_cache4_t *cache, bool to_cache, void *stream) {
  if (!d || !type_ok(d->type) || d->n_tokens < 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->rotary < 0 || d->rotary > d->head_dim ||
      d->max_position <= 0 || !(d->eps >= 0))
    return RNSWINO_E_INVALID;
  if (d->head_dim % 32 || d->head_dim > 256 || d->rotary % 16) return RNSWINO_E_UNSUPPORTED;
  const int64_t q_width = (int64_t)d->q_heads * d->head_dim, k_width = (int64_t)d->kv_heads * d->head_dim;
  if (q_width >= (1LL << 31) || k_width >= (1LL << 30)) return RNSWINO_E_UNSUPPORTED;
  // (which keeps the kernel's 32-bit numbers of heads in range too)
  if ((int64_t)d->n_tokens * (d->q_heads + (to_cache ? 2LL : 1LL) * d->kv_heads) > kMostThreads / rope_lanes(d->head_dim)) return RNSWINO_E_UNSUPPORTED;
  RopeArgs a = {};
  if (to_cache) {
    const int rc = cache_of(cache, a.cache);
    if (rc) return rc;
    if (a.cache.dim != d->head_dim || a.cache.heads != d->kv_heads) return RNSWINO_E_INVALID;
  }
  if (d->n_tokens == 0) return RNSWINO_OK;
  if (!rows_ok(q, d->q_stride, q_width) || !rows_ok(k, d->k_stride, k_width) || !rows_ok(q_out, d->q_out_stride, q_width) || !positions || (d->rotary && (!angles || !aligned(angles, 16))) ||
      (wq && !aligned(wq, 16)) || (wk && !aligned(wk, 16)))
    return RNSWINO_E_INVALID;
  if (to_cache ? !rows_ok(v, d->v_stride, k_width) || !slots : !rows_ok(k_out, d->k_out_stride, k_width)) return RNSWINO_E_INVALID;
  a.q = q, a.k = k, a.v = v, a.q_out = q_out, a.k_out = k_out, a.wq = wq, a.wk = wk, a.angles = angles, a.positions = positions, a.slots = slots;
  a.q_stride = d->q_stride, a.k_stride = d->k_stride, a.v_stride = d->v_stride, a.q_out_stride = d->q_out_stride, a.k_out_stride = d->k_out_stride;
  a.tokens = d->n_tokens, a.q_heads = d->q_heads, a.kv_heads = d->kv_heads, a.dim = d->head_dim, a.rotary = d->rotary, a.adjacent = d->adjacent != 0;
  a.max_position = d->max_position, a.eps = d->eps, a.inv_dim = 1.0f / (float)d->head_dim;
  if (d->type == RNSWINO_TYPE_BF16) to_cache ? launch_rope<Bf16, true>(a, (hipStream_t)stream) : launch_rope<Bf16, false>(a, (hipStream_t)stream);
  else to_cache ? launch_rope<F16, true>(a, (hipStream_t)stream) : launch_rope<F16, false>(a, (hipStream_t)stream);
  return launch_result();
}

// Tiles of 16 rows a wave of the kernel for many rows holds: as many as leave a SIMD two waves.
constexpr int many_tiles(int32_t type, int dim) { return dim <= 96 || (dim == 128 && type == RNSWINO_TYPE_BF16) ? 2 : 1; }
int many_rows(int32_t type, int dim) { return 64 * many_tiles(type, dim); }

// What an attention's description has to be; `a` gets its sizes and the launch.
int attention_of(const rnswino_cache4_t *cache, const rnswino_attention_t *d, AttendArgs &a) {
  a = {};
  const int rc = cache_of(cache, a.cache);
  if (rc) return rc;
  if (!d || !type_ok(d->type) || d->n_requests <= 0 || d->n_tokens < 0 || d->q_heads <= 0 || d->table_width <= 0 || d->window < 0 || d->max_fresh < 0 || d->max_len < 0 ||
      !(d->scale > 0) || d->scale > 1e30f || d->q_heads % a.cache.heads)
    return RNSWINO_E_INVALID;
  if (a.cache.dim != 64 && a.cache.dim != 96 && a.cache.dim != 128 && a.cache.dim != 256) return RNSWINO_E_UNSUPPORTED;
  a.group = d->q_heads / a.cache.heads;
  if (((int64_t)d->n_tokens + d->n_requests) * d->q_heads >= (1LL << 31)) return RNSWINO_E_UNSUPPORTED;
  if ((((int64_t)a.cache.pages * a.cache.heads) << a.cache.page_shift) >= (1LL << 32)) return RNSWINO_E_UNSUPPORTED;  // more rows than the card's memory holds
  if (((int64_t)d->table_width << a.cache.page_shift) > INT32_MAX - 4096) return RNSWINO_E_UNSUPPORTED;  // positions, those of the steps asked for ahead too, have 32 bits
  a.requests = d->n_requests, a.tokens = d->n_tokens, a.q_heads = d->q_heads, a.width = d->table_width, a.window = d->window;
  a.q_stride = d->q_stride, a.out_stride = d->out_stride;
  a.factor = d->scale * 1.44269504088896340736f;
  // no request has more new tokens than `fresh`, or more positions that a row sees than `len`
  const int64_t fresh = d->max_fresh && d->max_fresh < d->n_tokens ? d->max_fresh : d->n_tokens;
  int64_t len = (int64_t)d->table_width << a.cache.page_shift;
  if (d->max_len && d->max_len < len) len = d->max_len;
  if (d->window && d->window + fresh < len) len = d->window + fresh;
  const int64_t steps = (len + kAttendStep - 1) / kAttendStep;
  const auto tiles_of = [&](int rows) {  // that there are at most, of all heads
    const int64_t each = (fresh * a.group + rows - 1) / rows * d->n_requests, packed = (int64_t)d->n_tokens * a.group / rows + d->n_requests;
    return (each < packed ? each : packed) * a.cache.heads;
  };
  // The kernel for many rows does two to three times the products of the other in a second once it has a workgroup of eight steps for each of the 256 compute units (22 requests of 128 to 200
  // new tokens, 8 and 2 heads of 128: 274 workgroups 20.9 us, the other 28.8); with fewer the other's smaller tiles make up for it (seven requests of 300 rows of 64 dimensions, windows of 500:
  // 128 workgroups 20.8 us, the other 17.5).  With 256 dimensions, where a compute unit holds two of the other's instead of three, from half as many (one request of 165, 64 and 8 heads: 168
  // workgroups 14.5 us, the other 21.4).
  const int many = many_rows(d->type, a.cache.dim);
  const int64_t many_groups = tiles_of(many) * (steps < 8 ? 1 : steps / 8);
  a.tile_rows = fresh * a.group > 32 && many_groups >= (a.cache.dim == 256 ? 128 : 256) ? many : 16;
  a.tiles = fresh * a.group <= a.tile_rows ? d->n_requests : (int)((int64_t)d->n_tokens * a.group / a.tile_rows + d->n_requests);
  const int64_t real = tiles_of(a.tile_rows) > 1 ? tiles_of(a.tile_rows) : 1;
  int64_t splits = 1;
  // A tile is parted where its workgroups leave the card idle.  Few rows: joining takes 5 us, as long as a wave takes for six steps (24 of a workgroup; 24 requests of 736 positions, 48 units
  // of 11 steps: 9 us, parted 11.9), so parts have 16 steps (47 requests of 500 to 1949, 376 units: 19.8 us, five parts of 4 to 8 steps 23.2) unless there are few units for the card (one request of
  // 4001, 8 units: 13 parts of 5 steps 13.4 us, 3 of 21 steps 19.4).  2048 workgroups, so that requests of different lengths even out (64 requests of 500 to 16000, 512 units: four parts 72 us, two
  // 103); with many parts a tile they do so anyway, and three a compute unit run at once (6 requests of 20339, 48 units: 16 parts 23.2 us, 19 parts 25.5).
  // Many rows: two a compute unit run at once, and a part's sums cost more (15 requests of 165 to 300, 16 and 2 heads, 336 units: 66 us, in three parts 92).
  if (a.tile_rows == 16) {
    if (real < 768 && steps > 24) {
      splits = (real <= 48 ? 768 : 2048) / real;
      splits = splits < steps / 16 ? splits : steps / 16;
      if (real * splits < 256) splits = 256 / real < steps / kAttendWaves ? 256 / real : steps / kAttendWaves;
    }
  } else if (real < 512) {
    splits = 512 / real < steps / 4 ? 512 / real : steps / 4;
  }
  splits = splits < 64 ? splits : 64;
  splits = splits > 1 ? splits : 1;
  a.share = (int)((steps + splits - 1) / splits);
  a.splits = (int)((steps + a.share - 1) / a.share);
  return (int64_t)a.tiles * a.cache.heads * a.splits <= kMostThreads / (64 * kAttendWaves) ? RNSWINO_OK : RNSWINO_E_UNSUPPORTED;
}
int64_t attention_part_bytes(const AttendArgs &a) {
  return a.splits > 1 ? (int64_t)a.tiles * a.cache.heads * a.splits * part_floats(a.tile_rows, a.cache.dim) * 4 : 0;
}

template <typename T, int D>
void launch_attention(const AttendArgs &a, hipStream_t stream) {
  constexpr int kTiles = many_tiles(__is_same(T, F16) ? RNSWINO_TYPE_F16 : RNSWINO_TYPE_BF16, D);
  const unsigned units = (unsigned)a.tiles * a.cache.heads;
  if (a.tile_rows == 16) {
    hipLaunchKernelGGL((k_cache4_attend<T, D>), dim3(units * a.splits), dim3(64 * kAttendWaves), 0, stream, a);
    if (a.splits > 1) hipLaunchKernelGGL((k_cache4_join<T, D, 16>), dim3(units, 4), dim3(256), 0, stream, a);
  } else {
    hipLaunchKernelGGL((k_cache4_attend_many<T, D, kTiles>), dim3(units * a.splits), dim3(256), 0, stream, a);
    if (a.splits > 1) hipLaunchKernelGGL((k_cache4_join<T, D, 64 * kTiles>), dim3(units, 16 * kTiles), dim3(256), 0, stream, a);
  }
}
template <typename T>
void launch_attention(const AttendArgs &a, hipStream_t stream) {
  switch (a.cache.dim) {
    case 64: return launch_attention<T, 64>(a, stream);
    case 96: return launch_attention<T, 96>(a, stream);
    case 128: return launch_attention<T, 128>(a, stream);
    default: return launch_attention<T, 256>(a, stream);
  }
}

// ---- products in 8-bit floating point ----

int blocks_of(int32_t inputs) { return (int)(((int64_t)inputs + kBlock - 1) / kBlock); }
bool product_ok(int32_t n_rows, int32_t outputs, int32_t inputs) {
  return n_rows >= 0 && outputs > 0 && inputs > 0 && n_rows <= (1 << 22) && outputs <= (1 << 22) && inputs <= (1 << 22);
}
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T>
void launch_rows(const void *x, int64_t stride, int rows, int cols, uint8_t *codes, float *scales, hipStream_t stream) {
  const int blocks = blocks_of(cols);
  const int64_t groups = ((int64_t)rows * blocks + 15) / 16;
  const dim3 grid((unsigned)(groups < 65536 ? groups : 65536));
  hipLaunchKernelGGL(k_fp8_rows<T>, grid, dim3(256), 0, stream, (const uint16_t *)x, stride, rows, cols, blocks, codes, scales);
}

template <typename T, int WN, int WM, int RN, int RM, int STAGES>
void launch_many(const Fp8Args &a, hipStream_t stream) {
  const unsigned tiles = (unsigned)((a.outputs + 16 * WN * RN - 1) / (16 * WN * RN)) * (unsigned)((a.rows + 16 * WM * RM - 1) / (16 * WM * RM));
  hipLaunchKernelGGL((k_fp8_many<T, WN, WM, RN, RM, STAGES>), dim3((tiles + 7) / 8 * 8), dim3(64 * WN * WM), 0, stream, a);
}
template <typename T, int COLS, bool FROM_ROWS, int WAVES, int STAGES>
void launch_few(const Fp8Args &a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.outputs + 15) / 16), (unsigned)((a.rows + 16 * COLS - 1) / (16 * COLS)));
  hipLaunchKernelGGL((k_fp8_few<T, COLS, FROM_ROWS, WAVES, STAGES>), grid, dim3(64 * WAVES), 0, stream, a);
}
int64_t tiles_of(const Fp8Args &a, int outputs, int rows) { return (int64_t)((a.outputs + outputs - 1) / outputs) * ((a.rows + rows - 1) / rows); }

// Rows straight from 16-bit elements, each workgroup quantising its 16: where that takes no longer than a launch before it, which is with 16384 codes and up to two workgroups a compute unit (16 rows
// of 1024: 5.7 us, quantised before it 4.8 and 4.6; of 2048: 8.6, 4.8 and 4.6; 64 x 1778 x 1024, 448 workgroups: 6.8, and 4.7 and 4.7; 100 rows of the same, 784: 10.5, and 4.9 and 4.8).
bool from_rows(int32_t n_rows, int32_t outputs, int32_t blocks) {
  const int64_t codes = (int64_t)(n_rows < 16 ? n_rows : 16) * blocks * kBlock, groups = ((int64_t)outputs + 15) / 16 * (((int64_t)n_rows + 15) / 16);
  return codes <= kFewCodes && (n_rows <= 16 || groups <= 512);
}

// More than 16 rows have a workspace whichever way they go: what a caller has to bring grows with the rows alone.
bool no_workspace(int32_t n_rows, int32_t outputs, int32_t blocks) { return n_rows <= 16 && from_rows(n_rows, outputs, blocks); }

template <typename T>
void launch_product(const Fp8Args &a, hipStream_t stream) {
  // Few rows: the widest of k_fp8_few whose workgroups still come to one a compute unit, so that rows are read as seldom as that allows.  1000 outputs, 4600 inputs: 64 rows take 5.9 us by
  // 16 rows a workgroup (252), 8.0 by 64; 128 rows 10.5 by 16 (504), 7.3 by 32.
  const auto groups = [&](int rows) { return tiles_of(a, 16, rows); };
  if (a.inputs) launch_few<T, 1, true, 8, 2>(a, stream);
  else if (a.rows <= 16 || groups(16) <= 256) launch_few<T, 1, false, 8, 4>(a, stream);
  else if (a.rows <= 32 || groups(32) <= 256) launch_few<T, 2, false, 4, 4>(a, stream);
  else if (groups(64) <= 256) launch_few<T, 4, false, 4, 3>(a, stream);
  // More: tiles of 64 x 64 up to two a compute unit (4096 x 4096: 65 rows 14 us, by k_fp8_few 16; 512 rows 20, by 128 x 128 31; 1024 rows 34, by 128 x 128 30), of 256 x 256 from one a compute
  // unit (8192 x 2048, 2048 rows: 40 us, by 128 x 128 45; 4096 x 4096, 2048 rows, which are 128 tiles: 58, by 128 x 128 40).
  else if (tiles_of(a, 64, 64) <= 512) launch_many<T, 2, 2, 2, 2, 4>(a, stream);
  else if (tiles_of(a, 256, 256) < 256) launch_many<T, 2, 2, 4, 4, 2>(a, stream);
  else launch_many<T, 2, 4, 8, 4, 2>(a, stream);
}

}  // namespace

extern "C" {

int rnswino_block_tables(const int32_t *cached, const int32_t *fresh, int32_t n_requests, const int32_t *free_pages, int32_t n_free, int32_t page_size,
                         int32_t *table, int32_t table_width, int32_t *row_start, int32_t *lens, int64_t *slots, int32_t *positions, int32_t n_tokens,
                         int32_t *needed, void *stream) {
  if (!cached || !fresh || n_requests <= 0 || n_free < 0 || (n_free && !free_pages) || !table || table_width <= 0 || !row_start || !lens || n_tokens < 0 ||
      (n_tokens && (!slots || !positions)) || !needed)
    return RNSWINO_E_INVALID;
  if (!page_size_ok(page_size)) return RNSWINO_E_UNSUPPORTED;
  // Results lie apart from what is read and from each other: every workgroup reads all lengths while others write (the last step's lens as this step's cached is the call that comes to mind).
  const int64_t n = n_requests, t = n_tokens;
  const Range written[] = {{table, 4 * n * table_width}, {row_start, 4 * n + 4}, {lens, 4 * n}, {slots, 8 * t}, {positions, 4 * t}, {needed, 4}},
              read[] = {{cached, 4 * n}, {fresh, 4 * n}, {free_pages, 4LL * n_free}};
  for (const Range &w : written) {
    for (const Range &r : read)
      if (overlap(w, r)) return RNSWINO_E_INVALID;
    for (const Range &other : written)
      if (&other != &w && overlap(w, other)) return RNSWINO_E_INVALID;
  }
  // Few requests: four waves, a request a thread, 256 at a time (64 requests of one token: 2.6 us, with the other form 5.6; 405: 3.4 and 5.8, with prompts among them 4.4 and 6.4; 800: 6.3 and
  // 6.7; 1500: 8.0 and 7.0).  More: a thread's share of eight, so that 8192 are summed in one go (4099 of them: 9 us, in two 12.5).
  const bool few = n_requests <= 768;
  const int threads = few ? 256 : 1024;
  const TableArgs a = {cached, fresh, free_pages, table, row_start, lens, positions, needed, slots, n_requests, n_free, table_width, n_tokens, threads, log2_of(page_size)};
  const unsigned blocks = n_tokens ? (unsigned)(((int64_t)n_tokens + threads - 1) / threads) : 1u;
  if (few) hipLaunchKernelGGL((k_block_tables<256, 1>), dim3(blocks), dim3(256), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL((k_block_tables<1024, 8>), dim3(blocks), dim3(1024), 0, (hipStream_t)stream, a);
  return launch_result();
}

int rnswino_qk_norm_rope(const rnswino_rope_t *desc, const void *q, const void *k, const void *wq, const void *wk, const float *angles,
                         const int32_t *positions, void *q_out, void *k_out, void *stream) {
  return rope(desc, q, k, nullptr, wq, wk, angles, positions, nullptr, q_out, k_out, nullptr, false, stream);
}

int rnswino_qk_norm_rope_cache4(const rnswino_rope_t *desc, const void *q, const void *k, const void *v, const void *wq, const void *wk, const float *angles,
                                const int32_t *positions, const int64_t *slots, void *q_out, const rnswino_cache4_t *cache, void *stream) {
  return rope(desc, q, k, v, wq, wk, angles, positions, slots, q_out, nullptr, cache, true, stream);
}

int rnswino_cache4_read(const rnswino_cache4_t *cache, const int64_t *slots, int64_t n, int32_t type, void *k_out, void *v_out, void *stream) {
  Cache4 c;
  const int rc = cache_of(cache, c);
  if (rc) return rc;
  if (!type_ok(type) || n < 0) return RNSWINO_E_INVALID;
  if (n >= (1LL << 40) / ((int64_t)c.heads * c.dim)) return RNSWINO_E_UNSUPPORTED;
  if (n == 0) return RNSWINO_OK;
  if (!slots || !k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16)) return RNSWINO_E_INVALID;
  const int64_t blocks = (2 * n * c.heads * (c.dim / 8) + 255) / 256;
  const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536));
  if (type == RNSWINO_TYPE_BF16) hipLaunchKernelGGL(k_cache4_read<Bf16>, grid, dim3(256), 0, (hipStream_t)stream, c, slots, n, (uint16_t *)k_out, (uint16_t *)v_out);
  else hipLaunchKernelGGL(k_cache4_read<F16>, grid, dim3(256), 0, (hipStream_t)stream, c, slots, n, (uint16_t *)k_out, (uint16_t *)v_out);
  return launch_result();
}

size_t rnswino_cache4_attention_workspace_bytes(const rnswino_cache4_t *cache, const rnswino_attention_t *desc) {
  AttendArgs a;
  return attention_of(cache, desc, a) ? 0 : (size_t)attention_part_bytes(a);
}

int rnswino_cache4_attention(const rnswino_cache4_t *cache, const rnswino_attention_t *desc, const void *q, const int32_t *table, const int32_t *lens,
                             const int32_t *row_start, void *out, void *workspace, void *stream) {
  AttendArgs a;
  const int rc = attention_of(cache, desc, a);
  if (rc) return rc;
  if (a.tokens == 0) return RNSWINO_OK;
  const int64_t width = (int64_t)a.q_heads * a.cache.dim;
  if (!rows_ok(q, a.q_stride, width) || !rows_ok(out, a.out_stride, width) || !table || !lens || !row_start) return RNSWINO_E_INVALID;
  if (attention_part_bytes(a) && (!workspace || !aligned(workspace, 256))) return RNSWINO_E_INVALID;
  a.q = (const uint16_t *)q, a.out = (uint16_t *)out, a.table = table, a.lens = lens, a.row_start = row_start, a.part = (float *)workspace;
  if (desc->type == RNSWINO_TYPE_BF16) launch_attention<Bf16>(a, (hipStream_t)stream);
  else launch_attention<F16>(a, (hipStream_t)stream);
  return launch_result();
}

int rnswino_fp8_quantize_rows(const void *x, int32_t type, int32_t n_rows, int32_t inputs, int64_t stride, uint8_t *codes, float *scales, void *stream) {
  if (!type_ok(type) || n_rows < 0 || inputs <= 0 || stride < inputs) return RNSWINO_E_INVALID;
  if (!product_ok(n_rows, 1, inputs)) return RNSWINO_E_UNSUPPORTED;
  if (n_rows == 0) return RNSWINO_OK;
  if (!x || !aligned(x, 2) || !codes || !aligned(codes, 16) || !scales || !aligned(scales, 4)) return RNSWINO_E_INVALID;
  if (type == RNSWINO_TYPE_BF16) launch_rows<Bf16>(x, stride, n_rows, inputs, codes, scales, (hipStream_t)stream);
  else launch_rows<F16>(x, stride, n_rows, inputs, codes, scales, (hipStream_t)stream);
  return launch_result();
}

int rnswino_fp8_quantize_weights(const void *w, int32_t type, int32_t outputs, int32_t inputs, int64_t stride, uint8_t *codes, float *scales, void *stream) {
  if (!type_ok(type) || outputs <= 0 || inputs <= 0 || stride < inputs || !w || !aligned(w, 2) || !codes || !aligned(codes, 16) || !scales || !aligned(scales, 4))
    return RNSWINO_E_INVALID;
  if (!product_ok(1, outputs, inputs)) return RNSWINO_E_UNSUPPORTED;
  const int blocks = blocks_of(inputs);
  const dim3 grid((unsigned)blocks * (unsigned)blocks_of(outputs));
  if (type == RNSWINO_TYPE_BF16)
    hipLaunchKernelGGL(k_fp8_weights<Bf16>, grid, dim3(256), 0, (hipStream_t)stream, (const uint16_t *)w, stride, outputs, inputs, blocks, codes, scales);
  else hipLaunchKernelGGL(k_fp8_weights<F16>, grid, dim3(256), 0, (hipStream_t)stream, (const uint16_t *)w, stride, outputs, inputs, blocks, codes, scales);
  return launch_result();
}

size_t rnswino_fp8_matmul_workspace_bytes(int32_t n_rows, int32_t outputs, int32_t inputs) {
  (void)n_rows, (void)outputs, (void)inputs;
  return 0;
}

int rnswino_fp8_matmul(const uint8_t *x, const float *xs, const uint8_t *w, const float *ws, int32_t n_rows, int32_t outputs, int32_t inputs, int32_t type,
                       void *y, int64_t stride, void *workspace, void *stream) {
  if (!type_ok(type) || n_rows < 0 || outputs <= 0 || inputs <= 0 || stride < outputs) return RNSWINO_E_INVALID;
  if (!product_ok(n_rows, outputs, inputs)) return RNSWINO_E_UNSUPPORTED;
  if (n_rows == 0) return RNSWINO_OK;
  if (!x || !xs || !w || !ws || !y || !aligned(x, 16) || !aligned(w, 16) || !aligned(xs, 4) || !aligned(ws, 4) || !aligned(y, 2)) return RNSWINO_E_INVALID;
  (void)workspace;
  const Fp8Args a = {x, w, xs, ws, (uint16_t *)y, stride, 0, n_rows, outputs, blocks_of(inputs), 0};
  if (type == RNSWINO_TYPE_BF16) launch_product<Bf16>(a, (hipStream_t)stream);
  else launch_product<F16>(a, (hipStream_t)stream);
  return launch_result();
}

size_t rnswino_fp8_linear_workspace_bytes(int32_t n_rows, int32_t outputs, int32_t inputs) {
  if (!product_ok(n_rows, outputs, inputs)) return 0;
  const size_t blocks = (size_t)blocks_of(inputs);
  if (no_workspace(n_rows, outputs, (int32_t)blocks)) return 0;
  return up256((size_t)n_rows * blocks * kBlock) + up256((size_t)n_rows * blocks * 4) + rnswino_fp8_matmul_workspace_bytes(n_rows, outputs, inputs);
}

int rnswino_fp8_linear(const void *x, int64_t x_stride, const uint8_t *w, const float *ws, int32_t n_rows, int32_t outputs, int32_t inputs, int32_t type,
                       void *y, int64_t stride, void *workspace, void *stream) {
  if (!type_ok(type) || n_rows < 0 || outputs <= 0 || inputs <= 0 || x_stride < inputs || stride < outputs) return RNSWINO_E_INVALID;
  if (!product_ok(n_rows, outputs, inputs)) return RNSWINO_E_UNSUPPORTED;
  if (n_rows == 0) return RNSWINO_OK;
  if (!x || !w || !ws || !y || !aligned(x, 2) || !aligned(w, 16) || !aligned(ws, 4) || !aligned(y, 2)) return RNSWINO_E_INVALID;
  const size_t blocks = (size_t)blocks_of(inputs);
  if (!no_workspace(n_rows, outputs, (int32_t)blocks) && (!workspace || !aligned(workspace, 256))) return RNSWINO_E_INVALID;
  if (from_rows(n_rows, outputs, (int32_t)blocks)) {
    const Fp8Args a = {(const uint8_t *)x, w, nullptr, ws, (uint16_t *)y, stride, x_stride, n_rows, outputs, (int32_t)blocks, inputs};
    if (type == RNSWINO_TYPE_BF16) launch_product<Bf16>(a, (hipStream_t)stream);
    else launch_product<F16>(a, (hipStream_t)stream);
    return launch_result();
  }
  uint8_t *codes = (uint8_t *)workspace;
  float *scales = (float *)(codes + up256((size_t)n_rows * blocks * kBlock));
  const int rc = rnswino_fp8_quantize_rows(x, type, n_rows, inputs, x_stride, codes, scales, stream);
  if (rc) return rc;
  return rnswino_fp8_matmul(codes, scales, w, ws, n_rows, outputs, inputs, type, y, stride, (uint8_t *)scales + up256((size_t)n_rows * blocks * 4), stream);
}

}  // extern "C"
