// Shape functions, checks and the dispatch function of the paged cache's operators: host arithmetic only, no HIP call.
#include "cache_internal.h"

#include <cmath>

namespace nimble {

static bool misaligned(const void* p, unsigned to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

static int check_layout(int64_t pages, int64_t kv_heads, int64_t page, int64_t D, int dtype) {
  if (dtype != NIMBLE_BF16 && dtype != NIMBLE_I8) return fail(NIMBLE_ERR_DTYPE, "cache: dtype %d, bf16 or int8 needed", dtype);
  if (pages < 0 || kv_heads < 0 || page < 0 || D < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (D != 64 && D != 128) return fail(NIMBLE_ERR_ARG, "cache: heads of %lld, 64 or 128 needed", (long long)D);
  if (page < 16 || page > 1024 || (page & (page - 1))) return fail(NIMBLE_ERR_ARG, "cache: pages of %lld, a power of two from 16 to 1024 needed", (long long)page);
  if (kv_heads < 1 || kv_heads > 1024) return fail(NIMBLE_ERR_ARG, "cache: %lld heads, 1 to 1024 needed", (long long)kv_heads);
  if (pages > (1ll << 31) - 1) return fail(NIMBLE_ERR_ARG, "extent too large");
  return NIMBLE_OK;
}

int check_cache(const nimble_cache* c) {
  if (!c) return fail(NIMBLE_ERR_NULL, "null cache");
  const int rc = check_layout(c->pages, c->kv_heads, c->page, c->D, c->dtype);
  if (rc != NIMBLE_OK) return rc;
  if (c->pages == 0) return NIMBLE_OK;
  const bool int8 = c->dtype == NIMBLE_I8;
  if (!c->k || !c->v || (int8 && (!c->k_scale || !c->v_scale))) return fail(NIMBLE_ERR_NULL, "null cache pointer");
  if (misaligned(c->k) || misaligned(c->v) || (int8 && (misaligned(c->k_scale) || misaligned(c->v_scale))))
    return fail(NIMBLE_ERR_ALIGN, "device pointers must be 16-byte aligned");
  return NIMBLE_OK;
}

static int check_counts(int64_t rows, int64_t count, int64_t width, int64_t page) {
  if (rows < 0 || count < 0 || width < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (rows > kMostRows || count > kMostSequences) return fail(NIMBLE_ERR_ARG, "%lld rows of %lld sequences, at most %lld of %lld", (long long)rows, (long long)count,
                                                              (long long)kMostRows, (long long)kMostSequences);
  if (width > kMostPositions / page) return fail(NIMBLE_ERR_ARG, "page table of %lld pages of %lld: more than 2^30 positions", (long long)width, (long long)page);
  return NIMBLE_OK;
}

int check_sequences(const nimble_sequences* s, int64_t page) {
  if (!s) return fail(NIMBLE_ERR_NULL, "null sequences");
  const int rc = check_counts(s->rows, s->count, s->width, page);
  if (rc != NIMBLE_OK) return rc;
  if (s->rows == 0 || s->count == 0) return NIMBLE_OK;
  if (!s->offsets || !s->lengths || (s->width > 0 && !s->pages)) return fail(NIMBLE_ERR_NULL, "null sequences pointer");
  if (misaligned(s->offsets, 8) || misaligned(s->lengths, 8) || misaligned(s->pages, 4))
    return fail(NIMBLE_ERR_ALIGN, "offsets and lengths must be 8-byte aligned, pages 4-byte");
  return NIMBLE_OK;
}

// Rows that lie in each other's gaps share nothing; those of two strides are only taken for it where one lot lies behind the other.
static bool share(const Extent& a, const Extent& b) {
  if (!a.at || !b.at || a.rows <= 0 || b.rows <= 0 || a.bytes <= 0 || b.bytes <= 0) return false;
  typedef __int128 Wide;
  const Wide d = (Wide)(uintptr_t)b.at - (Wide)(uintptr_t)a.at;                        // of the first rows
  if (d >= (Wide)(a.rows - 1) * a.stride + a.bytes || -d >= (Wide)(b.rows - 1) * b.stride + b.bytes) return false;
  if (a.rows > 1 && b.rows > 1 && a.stride != b.stride) return true;
  const Wide stride = a.rows > 1 ? a.stride : b.stride;
  // rows i of a and j of b share bytes where d - a.bytes < (i - j) stride < d + b.bytes, -(b.rows - 1) <= i - j <= a.rows - 1
  Wide k = d - a.bytes;
  k = k >= 0 ? k / stride + 1 : -((-k - 1) / stride);                                  // the least i - j with more
  if (k < -(b.rows - 1)) k = -(b.rows - 1);
  return k <= a.rows - 1 && k * stride < d + b.bytes;
}

int check_apart(const char* what, std::initializer_list<Extent> outputs, std::initializer_list<Extent> operands) {
  for (const Extent* o = outputs.begin(); o != outputs.end(); ++o) {
    for (const Extent* x = o + 1; x != outputs.end(); ++x)
      if (share(*o, *x)) return fail(NIMBLE_ERR_ARG, "%s: %s and %s overlap", what, o->name, x->name);
    for (const Extent& x : operands)
      if (share(*o, x)) return fail(NIMBLE_ERR_ARG, "%s: %s and %s overlap", what, o->name, x.name);
  }
  return NIMBLE_OK;
}

// One after the other: keys, values and, in 8 bits, their scales; the batch's offsets, lengths and pages.
std::array<Extent, 4> cache_extents(const nimble_cache& c) {
  const int64_t slots = c.pages * c.kv_heads * c.page, element = c.dtype == NIMBLE_I8 ? 1 : 2, scale = c.dtype == NIMBLE_I8 ? 4 : 0;
  return {extent("the cache's keys", c.k, slots * c.D * element), extent("the cache's values", c.v, slots * c.D * element),
          extent("the keys' scales", c.k_scale, slots * scale), extent("the values' scales", c.v_scale, slots * scale)};
}
std::array<Extent, 3> sequences_extents(const nimble_sequences& s) {
  return {extent("offsets", s.offsets, (s.count + 1) * 8), extent("lengths", s.lengths, s.count * 8), extent("pages", s.pages, s.count * s.width * 4)};
}

CacheArgs cache_args(const nimble_cache& c) {
  CacheArgs a{(unsigned char*)c.k, (unsigned char*)c.v, (float*)c.k_scale, (float*)c.v_scale, (unsigned)c.pages, (int)c.kv_heads, 0};
  while ((1ll << a.page_shift) < c.page) ++a.page_shift;
  return a;
}

SequencesArgs sequences_args(const nimble_sequences& s) {
  return SequencesArgs{(const long long*)s.offsets, (const long long*)s.lengths, (const int*)s.pages, (int)s.count, (int)s.width, (int)s.rows};
}

// ------------------------------------------------------------------------------------------------ attention
constexpr int kPagedRows[NIMBLE_PAGED_COUNT] = {16, 128};
// Up to so many keys nothing is cut: the second launch costs more than a longer walk saves; half as many for few rows of bf16 heads of 128, which have four
// waves for a walk and not eight.  One token, cut / not, us:  16 heads of 64 in bf16 over 800 keys 10.0 / 8.4, 1200 10.4 / 10.3, 2000 10.2 / 12.8; in 8 bits 1000
// 10.0 / 10.2; 8 heads of 128 in 8 bits 800 11.3 / 11.2, 1000 11.4 / 12.6, in bf16 500 11.5 / 10.5, 800 11.6 / 13.7; of each of 64 sequences, 8 heads of 128
// in 8 bits, 1000 27.0 / 25.5.
constexpr int64_t kUncutKeys = 1024;
// Spans of few rows are counted in so many keys; in half as many where a tile has up to 4 rows, whose parts are joined by a workgroup a row, and even then no more
// spans than compute units, of up to 4096 keys, so that no row has more than 32 parts.  Microseconds, 256 / 128 keys a step: one token over 2000 keys, 32 heads of 128
// over 8, 12.3 / 11.6, over 4000 13.2 / 12.2, in 8 bits 11.1 / 10.8 and 12.2 / 11.7; 16 heads of 64 over 2000 in 8 bits 10.4 / 9.8.  Beyond: over 8000 keys 14.5 / 15.7, in
// 8 bits 13.2 / 14.2; of two sequences over 4000 in 8 bits 13.0 / 15.6; tiles of 8 rows, 16 heads of 64 in 8 bits, over 2000 11.1 / 11.5, over 4000 12.7 / 17.1, of 16
// rows 13.5 / 19.9; 64 tokens over up to 8192 98.9 / 100.2.
constexpr int64_t kStepKeys = 256;
// Waves of a workgroup, and workgroups that a compute unit holds at once, by their LDS (tokens) and registers: as many parts as fill the chip once
// are aimed at.  Tokens: four waves where workgroups share a compute unit, so that one loads while another joins its waves' sums and goes over to
// the next tile (64 tokens over up to 8192 keys in 8 bits, spans of two tiles: eight waves 114 us, twice four 106); eight where tiles are few and short and the
// walk over one is what takes its time (one token over 777 keys of 64: four 10.4, eight 7.8).  Of bf16 heads of 128 the LDS holds four waves.
struct PagedWaves {
  int waves, per_cu;
};
static int four_waves_per_cu(int64_t D, int dtype) { return (D == 128 ? 1 : 2) * (dtype == NIMBLE_I8 ? 2 : 1); }
static PagedWaves paged_waves(int kernel, int64_t D, int dtype, bool lone) {
  if (kernel == NIMBLE_PAGED_CHUNKS) return {4, D == 64 ? 3 : 2};
  const int four = four_waves_per_cu(D, dtype);
  return lone && four > 1 ? PagedWaves{8, four / 2} : PagedWaves{4, four};
}

// Which kernel.  16 rows a workgroup for up to 16 rows a sequence (32 of heads of 64 in 8 bits, where sequences and heads are many), and for more where nothing
// is cut and its tiles are about as many as the chip holds; else 128.  Microseconds, 16 / 128 rows a workgroup (graph replays; rows: of a sequence and a head of the cache):
//   bf16, heads of 64, 16 of the cache:  1 sequence, 128 rows over 628 keys 7.6 / 14.1, 512 over 1012 13 / 20; 16, 64 over 564 19 / 15, 128 over 628 34 / 17,
//     1 sequence, 32 rows over 4032 17 / 13, 128 over 4128 25 / 17, over 30128 153 / 38
//   bf16, 128, 8:  1, 128 over 532 11 / 17; 4, 12 / 17; 16, 41 / 19; 1, 32 over 4008 17 / 14, over 30008 51 / 31
//   int8, 64, 16:  16, 128 over 628 27 / 21; 4, 32 over 4032 25 / 25, over 30032 90 / 80, 128 over 4128 58 / 36; 64, 32 over 532 27 / 34, over 4032 159 / 190;
//     1, 32 over 4032 18 / 14
//   int8, 128, 8:  16, 128 over 532 25 / 25; 4, 32 over 4008 24 / 23, over 30008 85 / 79, 128 over 30032 226 / 102
// (On 560 shapes of 32 to 512 rows, 1 to 64 sequences of equal kind and up to 30512 keys the rule's choice takes 0.2 % longer than the better one; 1.5 times for 16 sequences of
// 32 rows over 30008 keys of 8 heads of 64 in 8 bits, 199 / 135, 1.14 times at most elsewhere.)
static int paged_kernel(int64_t rows, int64_t live, int64_t kv_heads, int64_t D, int dtype, int64_t keys) {
  if (keys <= kUncutKeys && (rows / kPagedRows[0] + live) * kv_heads <= kComputeUnits * 3 / 2 * four_waves_per_cu(D, dtype)) return NIMBLE_PAGED_TOKENS;
  const bool small = dtype == NIMBLE_I8 && D == 64 && live * kv_heads >= kComputeUnits / 4;
  return rows > (small ? 32 : 16) * live ? NIMBLE_PAGED_CHUNKS : NIMBLE_PAGED_TOKENS;
}

static int plan_paged(int64_t rows, int64_t count, int64_t width, int64_t heads, int64_t kv_heads, int64_t page, int64_t D, int dtype,
                      int64_t window, nimble_paged_plan* p) {
  int rc = check_layout(0, kv_heads, page, D, dtype);
  if (rc == NIMBLE_OK) rc = check_counts(rows, count, width, page);
  if (rc != NIMBLE_OK) return rc;
  if (heads < 1 || heads > 65536 || heads % kv_heads) return fail(heads < 1 || heads > 65536 ? NIMBLE_ERR_ARG : NIMBLE_ERR_SHAPE, "%lld query heads over %lld of the cache", (long long)heads, (long long)kv_heads);
  if (window < 0) return fail(NIMBLE_ERR_ARG, "negative window");
  if (window >= kMostPositions) window = 0;  // all
  nimble_paged_plan out{};
  if (rows == 0 || count == 0) {  // nothing is launched
    out.rows = kPagedRows[0];
    *p = out;
    return NIMBLE_OK;
  }
  const int64_t group = heads / kv_heads, live = count < rows ? count : rows;
  auto seen = [&](int64_t tile_rows) {  // the most keys that a tile can see
    const int64_t all = width * page;
    return window > 0 && window + tile_rows < all ? window + tile_rows : all;
  };
  out.kernel = paged_kernel(rows * group, live, kv_heads, D, dtype, seen(kPagedRows[0]));
  out.rows = kPagedRows[out.kernel];
  const int64_t tiles = rows * group / out.rows + live, keys = seen(out.rows);   // a sequence adds at most one tile that is not full
  const bool four = four_waves_per_cu(D, dtype) == 1 && rows * group <= kPagedRows[0] * live;
  out.parts = keys > (four ? kUncutKeys / 2 : kUncutKeys);
  const PagedWaves w = paged_waves(out.kernel, D, dtype, !out.parts && tiles * kv_heads <= kComputeUnits);
  const int64_t target = (int64_t)kComputeUnits * w.per_cu;
  out.block = 64u * (unsigned)w.waves;
  if (tiles * kv_heads > kMostPagedGrid) return fail(NIMBLE_ERR_ARG, "more than 2^23 tiles");
  if (tiles * kv_heads > ((1ll << 31) - 1) / (ceil_div(keys, kStepKeys) + 1))
    return fail(NIMBLE_ERR_ARG, "%lld tiles of %lld keys", (long long)(tiles * kv_heads), (long long)keys);
  if (out.parts) {
    // tokens: a span a workgroup, with two parts; chunks: a unit a workgroup, tiles and as many more as the cuts make
    const bool spans = out.kernel == NIMBLE_PAGED_TOKENS;
    const bool halves = rows * group <= 4 * live && keys <= 4096 && tiles * kv_heads * ceil_div(keys, kStepKeys / 2) <= kComputeUnits;
    out.step = (int32_t)(spans ? halves ? kStepKeys / 2 : kStepKeys : 0);
    out.grid = (uint32_t)(spans ? target : tiles * kv_heads + target);
    out.slots = 2 * target + 8;
    const int64_t most = rows * group < out.rows ? rows * group : out.rows;
    out.join_grid[0] = (uint32_t)(spans ? target : tiles * kv_heads < target ? tiles * kv_heads : target);
    const int64_t across = 2048 / out.join_grid[0] < 4 ? 4 : 2048 / out.join_grid[0];  // (few tiles: their rows side by side)
    out.join_grid[1] = (uint32_t)(most < across ? most : across);
    out.workspace_bytes = (uint64_t)out.slots * out.rows * (D * 4 + 8) + (uint64_t)(1 + target) * kPagedItemWords * 4;
  } else {
    out.grid = (uint32_t)(tiles * kv_heads);
  }
  *p = out;
  return NIMBLE_OK;
}

}  // namespace nimble

using namespace nimble;

extern "C" {

int nimble_rotary_shape(const int64_t* x_shape, int x_rank, const int64_t* positions_shape, int positions_rank, const int64_t* table_shape,
                        int table_rank, int64_t* out_shape) {
  clear_error();
  if (!x_shape || !positions_shape || !table_shape || !out_shape) return fail(NIMBLE_ERR_NULL, "null shape pointer");
  if (x_rank != 3 || positions_rank != 1 || table_rank != 3)
    return fail(NIMBLE_ERR_RANK, "rotary: ranks of x, positions, table are %d, %d, %d; 3, 1, 3 needed", x_rank, positions_rank, table_rank);
  for (int i = 0; i < 3; ++i)
    if (x_shape[i] < 0 || table_shape[i] < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (positions_shape[0] != x_shape[0])
    return fail(NIMBLE_ERR_SHAPE, "rotary: %lld positions for %lld rows", (long long)positions_shape[0], (long long)x_shape[0]);
  if (table_shape[2] != 2 || table_shape[1] > x_shape[2] / 2)
    return fail(NIMBLE_ERR_SHAPE, "rotary: a table of (%lld, %lld, %lld) for heads of %lld; (positions, pairs, 2) needed", (long long)table_shape[0],
                (long long)table_shape[1], (long long)table_shape[2], (long long)x_shape[2]);
  for (int i = 0; i < 3; ++i) out_shape[i] = x_shape[i];
  return NIMBLE_OK;
}

int nimble_cache_check(const int64_t* k_shape, int k_rank, const int64_t* v_shape, int v_rank, const int64_t* k_scale_shape,
                       int k_scale_rank, const int64_t* v_scale_shape, int v_scale_rank, int dtype, const int64_t* offsets_shape,
                       int offsets_rank, const int64_t* lengths_shape, int lengths_rank, const int64_t* pages_shape, int pages_rank) {
  clear_error();
  const bool int8 = dtype == NIMBLE_I8;
  if (!k_shape || !v_shape || !offsets_shape || !lengths_shape || !pages_shape || (int8 && (!k_scale_shape || !v_scale_shape)))
    return fail(NIMBLE_ERR_NULL, "null shape pointer");
  if (k_rank != 4 || v_rank != 4 || (int8 && (k_scale_rank != 3 || v_scale_rank != 3)))
    return fail(NIMBLE_ERR_RANK, "cache: keys and values of rank 4 and scales of rank 3 needed");
  if (offsets_rank != 1 || lengths_rank != 1 || pages_rank != 2)
    return fail(NIMBLE_ERR_RANK, "sequences: ranks of offsets, lengths, pages are %d, %d, %d; 1, 1, 2 needed", offsets_rank, lengths_rank, pages_rank);
  const int rc = check_layout(k_shape[0], k_shape[1], k_shape[2], k_shape[3], dtype);
  if (rc != NIMBLE_OK) return rc;
  for (int i = 0; i < 4; ++i)
    if (v_shape[i] != k_shape[i]) return fail(NIMBLE_ERR_SHAPE, "cache: keys and values differ in extent %d", i);
  for (int i = 0; int8 && i < 3; ++i)
    if (k_scale_shape[i] != k_shape[i] || v_scale_shape[i] != k_shape[i]) return fail(NIMBLE_ERR_SHAPE, "cache: scales differ from the codes in extent %d", i);
  if (lengths_shape[0] < 0 || pages_shape[0] < 0 || pages_shape[1] < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (offsets_shape[0] != lengths_shape[0] + 1 || pages_shape[0] != lengths_shape[0])
    return fail(NIMBLE_ERR_SHAPE, "sequences: %lld offsets and %lld rows of pages for %lld lengths", (long long)offsets_shape[0], (long long)pages_shape[0],
                (long long)lengths_shape[0]);
  return check_counts(0, lengths_shape[0], pages_shape[1], k_shape[2]);
}

int nimble_cache_write_shape(const int64_t* cache_shape, const int64_t* k_shape, int k_rank, const int64_t* v_shape, int v_rank,
                             const int64_t* q_shape, int q_rank, int64_t* q_out_shape) {
  clear_error();
  if (!cache_shape || !k_shape || !v_shape || (q_rank && (!q_shape || !q_out_shape))) return fail(NIMBLE_ERR_NULL, "null shape pointer");
  if (k_rank != 3 || v_rank != 3 || (q_rank && q_rank != 3))
    return fail(NIMBLE_ERR_RANK, "cache_write: ranks of k, v, q are %d, %d, %d; 3 needed", k_rank, v_rank, q_rank);
  for (int i = 0; i < 3; ++i) {
    if (k_shape[i] < 0 || v_shape[i] < 0 || (q_rank && q_shape[i] < 0)) return fail(NIMBLE_ERR_ARG, "negative extent");
    if (k_shape[i] != v_shape[i]) return fail(NIMBLE_ERR_SHAPE, "cache_write: keys and values differ in extent %d", i);
  }
  if (k_shape[1] != cache_shape[1] || k_shape[2] != cache_shape[3])
    return fail(NIMBLE_ERR_SHAPE, "cache_write: %lld heads of %lld for a cache of %lld of %lld", (long long)k_shape[1], (long long)k_shape[2],
                (long long)cache_shape[1], (long long)cache_shape[3]);
  if (!q_rank) return NIMBLE_OK;
  if (q_shape[0] != k_shape[0] || q_shape[2] != k_shape[2])
    return fail(NIMBLE_ERR_SHAPE, "cache_write: queries (%lld, ., %lld), keys (%lld, ., %lld)", (long long)q_shape[0], (long long)q_shape[2],
                (long long)k_shape[0], (long long)k_shape[2]);
  for (int i = 0; i < 3; ++i) q_out_shape[i] = q_shape[i];
  return NIMBLE_OK;
}

int nimble_cache_read_shape(const int64_t* cache_shape, int64_t rows, int64_t* out_shape) {
  clear_error();
  if (!cache_shape || !out_shape) return fail(NIMBLE_ERR_NULL, "null shape pointer");
  if (rows < 0 || cache_shape[1] < 0 || cache_shape[3] < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  out_shape[0] = rows;
  out_shape[1] = cache_shape[1];
  out_shape[2] = cache_shape[3];
  return NIMBLE_OK;
}

int nimble_paged_attention_shape(const int64_t* q_shape, int q_rank, const int64_t* cache_shape, int64_t* out_shape) {
  clear_error();
  if (!q_shape || !cache_shape || !out_shape) return fail(NIMBLE_ERR_NULL, "null shape pointer");
  if (q_rank != 3) return fail(NIMBLE_ERR_RANK, "paged_attention: q has rank %d, 3 needed", q_rank);
  for (int i = 0; i < 3; ++i)
    if (q_shape[i] < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (q_shape[2] != cache_shape[3]) return fail(NIMBLE_ERR_SHAPE, "paged_attention: heads of %lld, of the cache %lld", (long long)q_shape[2], (long long)cache_shape[3]);
  if (q_shape[1] < 1 || cache_shape[1] < 1 || q_shape[1] % cache_shape[1])
    return fail(NIMBLE_ERR_SHAPE, "paged_attention: %lld query heads over %lld of the cache", (long long)q_shape[1], (long long)cache_shape[1]);
  for (int i = 0; i < 3; ++i) out_shape[i] = q_shape[i];
  return NIMBLE_OK;
}

int nimble_paged_attention_plan_of(int64_t rows, int64_t count, int64_t width, int64_t heads, int64_t kv_heads, int64_t page, int64_t D,
                                   int dtype, int64_t window, nimble_paged_plan* plan) {
  clear_error();
  if (!plan) return fail(NIMBLE_ERR_NULL, "null plan pointer");
  return plan_paged(rows, count, width, heads, kv_heads, page, D, dtype, window, plan);
}

}  // extern "C"
