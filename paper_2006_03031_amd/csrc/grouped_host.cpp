// Shape functions and the dispatch function of the 8-bit and the grouped products: host arithmetic only, no HIP call.
#include "grouped_internal.h"

#include <cmath>

namespace nimble {

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The members of the family that need rows of whole 16 bytes: tile, waves among which K is divided, stages that are loaded ahead (large tiles);
// microseconds of a workgroup that do not depend on K (launch, first loads, sums and stores; of a large tile its end); KB per us at which a
// compute unit's stages arrive (streaming), or microseconds of a stage of 128 bytes of K on a full chip (large tiles).
struct Member {
  int kernel, bm, bn, k_waves, ahead;
  double fixed_us, rate;
};
static const Member kMembers[] = {
    {NIMBLE_PRODUCT_STREAM, 8, 32, 4, 0, 2.0, 66},    {NIMBLE_PRODUCT_STREAM, 16, 32, 4, 0, 2.0, 75},
    {NIMBLE_PRODUCT_STREAM, 32, 32, 4, 0, 2.2, 100},  {NIMBLE_PRODUCT_STREAM, 64, 64, 4, 0, 4.3, 93},
    {NIMBLE_PRODUCT_STREAM, 64, 64, 2, 0, 3.5, 56},   {NIMBLE_PRODUCT_TILES, 128, 256, 1, 3, 2.3, 0.78},
    {NIMBLE_PRODUCT_TILES, 160, 256, 1, 2, 3.1, 0.86}, {NIMBLE_PRODUCT_TILES, 192, 256, 1, 2, 2.8, 1.05},
    {NIMBLE_PRODUCT_TILES, 224, 256, 1, 2, 3.5, 1.15}, {NIMBLE_PRODUCT_TILES, 256, 256, 1, 2, 3.8, 1.25},
};

// Workgroups of a streaming member that share a compute unit, by their LDS: three of 8 x 32, two of 32 x 32 and of 64 x 64 by two waves, one of
// 64 x 64 by four; of 16 x 32 three without groups (49920 bytes each), two with the map of the groups (58120).
// (With three for either, 84 of 4000 grouped draws took 16 x 32 in what was thought to be fewer rounds, and 14 % longer on average.)
static int stream_workgroups_per_cu(const ProductShape& s, const Member& m) {
  return kComputeUnitLds / stream_lds_bytes(m.bm, m.bn, m.k_waves, kStreamStages, s.grouped ? kMostGroups : 0);
}

// The most tile rows there can be: a group adds at most one that is not full, and only if it has a row.
static int64_t most_tile_rows(const ProductShape& s, int bm) {
  return s.grouped ? s.rows / bm + (s.groups < s.rows ? s.groups : s.rows) : ceil_div(s.rows, bm);
}

// Estimated microseconds.  How the rows fall on the groups is not known: each group is taken to have rows where there are
// enough, and its last tile to be half full.  The workgroups of a compute unit share the rate at which stages arrive.  Large tiles go
// round the chip, on a nearly empty one (less power) with stages a third shorter; groups may have a few tiles more than that.
// Weights come at 4.8 TB/s where they come from memory, and then a quarter of the estimate still tells the members apart.
// The constants are a fit to the members' times, measured until the clocks have settled, on 400 shapes of either type (K = 128 .. 8192,
// N = 128 .. 8192, 1 .. 16354 rows over 1 .. 64 groups), 54 large ones and 27 of wide layers, where the choice costs 2.4, 0.4 and 1.6 % more than
// the best member; on 200 others it costs 2.9 %, on 36 other large ones 2.4 %.  (Fitted to short runs alone, large ones took 128 x 256 and 5 to 10 %
// longer.)  Dense in 8 bits with bias, us:
//   rows x N x K         8 x 32   32 x 32   64 x 64, 4 waves  64 x 64, 2 waves  128 x 256   192 x 256   256 x 256
//   1 x 4096 x 1024      2.9      3.3       6.0               6.3               10.1        12.1        14.8
//   200 x 1024 x 4096    9.9      5.3       9.1               13.3              25.4        32.5        40.3
//   512 x 1024 x 4096    19.5     9.4       10.6              13.8              26.2        33.1        41.3
//   512 x 4096 x 1024    30.2     13.8      11.6              9.1               10.8        13.1        16.1
//   8192 x 1024 x 4096                      79.2              65.4              31.5        34.6        42.0
//   16384 x 1024 x 4096                     152               129               60.6        69.1        53.0
//   8192 x 4096 x 1024                      163               117               40.7        40.0        34.9
//   8192 x 8192 x 8192                      1091              1070              463         441         397
static double product_us(const ProductShape& s, const Member& m) {
  const double kCUs = kComputeUnits;
  const double live = s.grouped ? (double)(s.groups < s.rows ? s.groups : s.rows) : 1.0;
  double tile_rows = s.grouped ? (double)s.rows / m.bm + 0.5 * live : (double)ceil_div(s.rows, m.bm);
  if (tile_rows < live) tile_rows = live;
  const double tiles = tile_rows * (double)ceil_div(s.N, m.bn), stages = (double)ceil_div(s.row_bytes(), 128);
  double us;
  if (m.kernel == NIMBLE_PRODUCT_TILES) {
    const double full = tiles < kCUs ? tiles / kCUs : 1.0;
    const double walk = (stages < m.ahead ? m.ahead : stages) * m.rate * (0.62 + 0.38 * full);
    us = 3.7 + ceil(tiles * (s.grouped && s.groups > 1 ? 1.03 : 1.0) / kCUs) * (walk + m.fixed_us);
  } else {
    const double per_cu = tiles < kCUs ? 1.0 : tiles / kCUs;
    us = 1.0 + ceil(tiles / (kCUs * stream_workgroups_per_cu(s, m))) * m.fixed_us + per_cu * stages * (m.bm + m.bn) * 0.128 / m.rate;
  }
  const double weights_us = live * (double)s.N * (double)s.row_bytes() / 4.8e6;
  return (us > weights_us ? us : weights_us) + 0.25 * us;
}

int plan_product(const ProductShape& s, nimble_product_plan* p) {
  nimble_product_plan out{};
  const int64_t rb = s.row_bytes();
  const Member* best = nullptr;
  double best_us = 0;
  if (rb % 16 == 0 && rb > 0 && rb <= kMostTileRowBytes) {
    for (const Member& m : kMembers) {
      if (m.kernel == NIMBLE_PRODUCT_TILES && (s.N % 8 != 0 || s.N > kMostTileColumns)) continue;  // (rows are stored in whole 16 bytes)
      const double us = product_us(s, m);
      if (!best || us < best_us) best = &m, best_us = us;
    }
  }
  if (best) {
    out.kernel = best->kernel;
    out.bm = best->bm;
    out.bn = best->bn;
    out.k_waves = best->k_waves;
    out.block = best->kernel == NIMBLE_PRODUCT_TILES ? 256 : 64u * (unsigned)best->k_waves;
  } else {
    // 16 x 16 tiles where a group has no more than 16 rows or the chip holds all of them at once: 64 x 4096 x 1003 in 8 bits 8.4 us, in 64 x 64
    // 10.9; 200 x 1024 x 4099 21.8 / 27.5; beyond that 512 x 1024 x 4096 35 / 20
    const int64_t live = s.grouped ? (s.groups < s.rows ? s.groups : s.rows) : 1;
    const bool few = s.rows <= 16 * live || most_tile_rows(s, 16) * ceil_div(s.N, 16) <= 4 * kComputeUnits;
    out.kernel = NIMBLE_PRODUCT_DIRECT;
    out.bm = out.bn = few ? 16 : 64;
    out.k_waves = few ? 8 : 4;
    out.block = 64u * (unsigned)out.k_waves;
  }
  const int64_t tile_rows = most_tile_rows(s, out.bm), tiles_n = ceil_div(s.N, out.bn);
  if (tile_rows > 0x7fffffffll / (tiles_n > 0 ? tiles_n : 1)) return fail(NIMBLE_ERR_ARG, "more than 2^31 tiles");
  out.tiles = tile_rows * tiles_n;
  // the large tiles' workgroups go round; the others' do where a launch could not hold them
  const int64_t most = out.kernel == NIMBLE_PRODUCT_TILES ? kComputeUnits : kMostWorkgroups;
  out.grid = (uint32_t)(out.tiles < most ? out.tiles : most);
  *p = out;
  return NIMBLE_OK;
}

static int check_product(int64_t R, int64_t E, int64_t N, int64_t K, bool int8) {
  if (R < 0 || E < 0 || N < 0 || K < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (E > kMostGroups) return fail(NIMBLE_ERR_ARG, "%lld groups, at most %d", (long long)E, kMostGroups);
  if (int8 && K > kMostK8) return fail(NIMBLE_ERR_ARG, "K = %lld: 32-bit sums of 8-bit products hold for K <= %lld", (long long)K, (long long)kMostK8);
  if (K > kMostK16 || N > (1ll << 30) || R > (1ll << 31) - 1) return fail(NIMBLE_ERR_ARG, "extent too large");
  return NIMBLE_OK;
}

}  // namespace nimble

using namespace nimble;

extern "C" {

int nimble_quantize_rows_shape(const int64_t* x_shape, int x_rank, int64_t cols, int64_t* q_shape, int64_t* scale_shape) {
  clear_error();
  if (!x_shape || !q_shape || !scale_shape) return fail(NIMBLE_ERR_NULL, "null shape pointer");
  if (x_rank != 2) return fail(NIMBLE_ERR_RANK, "quantize_rows: x has rank %d, 2 needed", x_rank);
  if (x_shape[0] < 0 || x_shape[1] < 0 || cols < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (x_shape[1] > (1ll << 30) || cols > (1ll << 30)) return fail(NIMBLE_ERR_ARG, "extent too large");
  if (cols == 0) cols = ceil_div(x_shape[1], 128) * 128;
  if (cols < x_shape[1])
    return fail(NIMBLE_ERR_SHAPE, "quantize_rows: %lld columns for rows of %lld", (long long)cols, (long long)x_shape[1]);
  q_shape[0] = scale_shape[0] = x_shape[0];
  q_shape[1] = cols;
  return NIMBLE_OK;
}

int nimble_dense_i8_shape(const int64_t* x_shape, int x_rank, const int64_t* x_scale_shape, int x_scale_rank, const int64_t* w_shape,
                          int w_rank, const int64_t* w_scale_shape, int w_scale_rank, int64_t* out_shape) {
  clear_error();
  if (!x_shape || !x_scale_shape || !w_shape || !w_scale_shape || !out_shape) return fail(NIMBLE_ERR_NULL, "null shape pointer");
  if (x_rank != 2 || w_rank != 2 || x_scale_rank != 1 || w_scale_rank != 1)
    return fail(NIMBLE_ERR_RANK, "dense_i8: ranks of x, x_scale, w, w_scale are %d, %d, %d, %d; 2, 1, 2, 1 needed", x_rank, x_scale_rank,
                w_rank, w_scale_rank);
  for (int i = 0; i < 2; ++i)
    if (x_shape[i] < 0 || w_shape[i] < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (x_shape[1] != w_shape[1])
    return fail(NIMBLE_ERR_SHAPE, "dense_i8: K of x is %lld, of w %lld", (long long)x_shape[1], (long long)w_shape[1]);
  if (x_scale_shape[0] != x_shape[0] || w_scale_shape[0] != w_shape[0])
    return fail(NIMBLE_ERR_SHAPE, "dense_i8: %lld and %lld scales for %lld and %lld rows", (long long)x_scale_shape[0],
                (long long)w_scale_shape[0], (long long)x_shape[0], (long long)w_shape[0]);
  out_shape[0] = x_shape[0];
  out_shape[1] = w_shape[0];
  return NIMBLE_OK;
}

int nimble_grouped_dense_shape(const int64_t* x_shape, int x_rank, const int64_t* w_shape, int w_rank, const int64_t* offsets_shape,
                               int offsets_rank, int64_t* out_shape) {
  clear_error();
  if (!x_shape || !w_shape || !offsets_shape || !out_shape) return fail(NIMBLE_ERR_NULL, "null shape pointer");
  if (x_rank != 2 || w_rank != 3 || offsets_rank != 1)
    return fail(NIMBLE_ERR_RANK, "grouped dense: ranks of x, w, offsets are %d, %d, %d; 2, 3, 1 needed", x_rank, w_rank, offsets_rank);
  if (x_shape[0] < 0 || x_shape[1] < 0 || w_shape[0] < 0 || w_shape[1] < 0 || w_shape[2] < 0)
    return fail(NIMBLE_ERR_ARG, "negative extent");
  if (x_shape[1] != w_shape[2])
    return fail(NIMBLE_ERR_SHAPE, "grouped dense: K of x is %lld, of w %lld", (long long)x_shape[1], (long long)w_shape[2]);
  if (offsets_shape[0] != w_shape[0] + 1)
    return fail(NIMBLE_ERR_SHAPE, "grouped dense: %lld offsets for %lld groups", (long long)offsets_shape[0], (long long)w_shape[0]);
  out_shape[0] = x_shape[0];
  out_shape[1] = w_shape[1];
  return NIMBLE_OK;
}

int nimble_product_plan_of(int64_t R, int64_t E, int64_t N, int64_t K, int in_dtype, int out_dtype, nimble_product_plan* plan) {
  clear_error();
  if (!plan) return fail(NIMBLE_ERR_NULL, "null plan pointer");
  if ((in_dtype != NIMBLE_BF16 && in_dtype != NIMBLE_I8) || (out_dtype != NIMBLE_BF16 && out_dtype != NIMBLE_F32))
    return fail(NIMBLE_ERR_DTYPE, "unknown dtype %d or %d", in_dtype, out_dtype);
  const bool grouped = E != -1, int8 = in_dtype == NIMBLE_I8;
  if (!grouped && !int8) return fail(NIMBLE_ERR_ARG, "bf16 without groups is nimble_dense_plan's");
  const int rc = check_product(R, grouped ? E : 1, N, K, int8);
  if (rc != NIMBLE_OK) return rc;
  return plan_product(ProductShape{R, grouped ? E : 1, N, K, grouped, int8, out_dtype == NIMBLE_F32}, plan);
}

}  // extern "C"
