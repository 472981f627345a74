// Shape functions and the dispatch function of the 8-bit and the grouped products.  Integer arithmetic only; no HIP call.
#include "grouped_internal.h"

#include <cstdlib>
#include <cstdio>

namespace nimble {

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int plan_product(const ProductShape& s, nimble_product_plan* p) {
  nimble_product_plan out{};
  const int64_t rb = s.row_bytes(), ks = ceil_div(rb, 128);
  const bool tiles_ok = rb % 16 == 0 && rb <= kMostTileRowBytes && s.N <= kMostTileColumns && s.N % 8 == 0 && (rb % 128 == 0 ? ks >= 3 : ks >= 4);
  const int64_t most_groups = s.grouped ? s.groups : 1;
  static const char* fs = getenv("PRODUCT");  // k,bm
  int fk = -1, fb = 0;
  if (fs) sscanf(fs, "%d,%d", &fk, &fb);
  int64_t most = kMostWorkgroups;
  const bool stream_ok = rb % 16 == 0 && rb > 0 && rb <= kMostTileRowBytes;
  if (fk == 1 ? tiles_ok : fk < 0 && tiles_ok && s.rows >= 256 * most_groups) {
    out.kernel = NIMBLE_PRODUCT_TILES;
    out.bm = 128;
    out.bn = 256;
    out.k_waves = 1;
    out.block = 256;
    most = 256;
  } else if (stream_ok && fk != 0) {
    out.kernel = NIMBLE_PRODUCT_STREAM;
    out.bm = out.bn = fb ? fb : s.rows <= 16 * most_groups ? 16 : s.rows <= 64 * most_groups ? 32 : 64;
    out.k_waves = 4;
    out.block = 256;
  } else {
    out.kernel = NIMBLE_PRODUCT_DIRECT;
    out.bm = fb ? fb : s.rows <= 16 * most_groups ? 16 : 64;
    out.bn = out.bm;
    out.k_waves = out.bm == 16 ? 8 : 4;
    out.block = 64u * (unsigned)out.k_waves;
  }
  // a group adds at most one tile row that is not full, and only if it has a row
  const int64_t tile_rows = s.grouped ? s.rows / out.bm + (s.groups < s.rows ? s.groups : s.rows) : ceil_div(s.rows, out.bm);
  const int64_t tiles_n = ceil_div(s.N, out.bn);
  if (tile_rows > 0x7fffffffll / (tiles_n > 0 ? tiles_n : 1)) return fail(NIMBLE_ERR_ARG, "more than 2^31 tiles");
  out.tiles = tile_rows * tiles_n;
  out.grid = (uint32_t)(out.tiles < most ? out.tiles : most);
  *p = out;
  return NIMBLE_OK;
}

static int check_product(int64_t R, int64_t E, int64_t N, int64_t K, bool grouped, bool int8) {
  if (R < 0 || E < 0 || N < 0 || K < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (E > kMostGroups) return fail(NIMBLE_ERR_ARG, "%lld groups, at most %d", (long long)E, kMostGroups);
  if (int8 && K > kMostK8) return fail(NIMBLE_ERR_ARG, "K = %lld: 32-bit sums of 8-bit products hold for K <= %lld", (long long)K, (long long)kMostK8);
  if (K > kMostK16 || N > (1ll << 30) || R > (1ll << 31) - 1) return fail(NIMBLE_ERR_ARG, "extent too large");
  (void)grouped;
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
  const int rc = check_product(R, grouped ? E : 1, N, K, grouped, int8);
  if (rc != NIMBLE_OK) return rc;
  return plan_product(ProductShape{R, grouped ? E : 1, N, K, grouped, int8, out_dtype == NIMBLE_F32}, plan);
}

}  // extern "C"
