// Device entry points of rotary positions and of the paged cache's reads and writes (kernels: cache_kernel.h).
#include <hip/hip_runtime.h>

#include <cmath>

#include "cache_kernel.h"
#include "grouped_internal.h"

namespace nimble {

int check_hip_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? NIMBLE_OK : fail(NIMBLE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}
static bool misaligned(const void* p, unsigned to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }
static dim3 grid_of(int64_t items, int64_t per) {
  const int64_t groups = ceil_div(items, per);
  return dim3((unsigned)(groups < kMostWorkgroups ? groups : kMostWorkgroups));
}

// Rows of `heads` heads of D elements, `stride` apart: the form that the cache's operators read.
int check_rows(const void* p, int64_t stride, int64_t heads, int64_t D, const char* what) {
  if (!p) return fail(NIMBLE_ERR_NULL, "null tensor pointer");
  if (misaligned(p)) return fail(NIMBLE_ERR_ALIGN, "device pointers must be 16-byte aligned");
  if (stride < heads * D || stride % 8) return fail(NIMBLE_ERR_ARG, "%s: rows of %lld elements, %lld apart: a multiple of 8 that holds a row is needed", what,
                                                    (long long)(heads * D), (long long)stride);
  return NIMBLE_OK;
}

// Rows of a workgroup: as many as leave each compute unit `groups` of them.
static int rows_each(int64_t rows, int groups) {
  const int64_t n = rows / (groups * kComputeUnits);
  return (int)(n < 1 ? 1 : n > kMostPlaces ? kMostPlaces : n);
}

// Workgroups for `rows` rows, rows_each of which take `lanes` lanes: where there are few, one for every 256 lanes (61 rows of 32 + 8 + 8 heads of 128 written
// into 8 bits: 4.7 -> 4.1 us; 200 rows of 64 + 32 + 32 8.3 -> 5.8, with half the workgroups 6.5; 64 rows of 32 heads of 128 read back 3.5 -> 2.6).
static dim3 grid_of_rows(int64_t rows, int64_t rows_each, int64_t lanes) {
  const int64_t x = ceil_div(rows, rows_each), room = 4 * kComputeUnits / x, y = ceil_div(lanes, 256) < room ? ceil_div(lanes, 256) : room;
  return dim3((unsigned)x, y > 1 ? (unsigned)y : 1);
}

template <int D, bool INTERLEAVED>
static void launch_write(const CacheWriteArgs& g, bool int8, hipStream_t stream) {
  const dim3 grid = grid_of_rows(g.seqs.rows, g.rows_each, (int64_t)g.rows_each * ((g.q ? g.heads : 0) + 2 * g.cache.kv_heads) * (D / 16)), block(256);
  if (int8)
    hipLaunchKernelGGL((cache_write_kernel<D, true, INTERLEAVED>), grid, block, 0, stream, g);
  else
    hipLaunchKernelGGL((cache_write_kernel<D, false, INTERLEAVED>), grid, block, 0, stream, g);
}

template <int D>
static void launch_read(const CacheReadArgs& g, bool int8, bool f32, hipStream_t stream) {
  const dim3 grid = grid_of_rows(g.seqs.rows, g.rows_each, (int64_t)g.rows_each * 2 * g.cache.kv_heads * (D / 8)), block(256);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, g); };
  if (int8) {
    if (f32) launch(cache_read_kernel<D, true, true>);
    else launch(cache_read_kernel<D, true, false>);
  } else {
    if (f32) launch(cache_read_kernel<D, false, true>);
    else launch(cache_read_kernel<D, false, false>);
  }
}

}  // namespace nimble

using namespace nimble;

extern "C" {

int nimble_rotary_table_dyn(void* table, int64_t positions, int64_t rot, double base, double factor, double trained, double low,
                            double high, double magnitude, void* stream) {
  clear_error();
  if (positions < 0 || rot < 0 || rot % 2) return fail(NIMBLE_ERR_ARG, "rotary_table: %lld positions of %lld elements, an even number needed", (long long)positions, (long long)rot);
  if (positions > (1ll << 31) || rot > (1 << 20)) return fail(NIMBLE_ERR_ARG, "extent too large");
  if (!(base > 0 && factor > 0 && high > low && trained >= 0) || !std::isfinite(base) || !std::isfinite(factor) || !std::isfinite(trained) ||
      !std::isfinite(low) || !std::isfinite(high) || !std::isfinite(magnitude))
    return fail(NIMBLE_ERR_ARG, "rotary_table: base, factor > 0, high > low, trained >= 0, all finite needed");
  const int64_t count = positions * (rot / 2);
  if (count == 0) return NIMBLE_OK;
  if (!table) return fail(NIMBLE_ERR_NULL, "null tensor pointer");
  if (misaligned(table)) return fail(NIMBLE_ERR_ALIGN, "device pointers must be 16-byte aligned");
  hipLaunchKernelGGL(rotary_table_kernel, grid_of(count, 256), dim3(256), 0, (hipStream_t)stream, (float2*)table, (long long)count, (int)(rot / 2), base,
                     factor, trained, low, high, magnitude);
  return check_hip_launch("rotary table kernel launch");
}

int nimble_rotary_dyn(const void* x, int64_t x_stride, const void* positions, const void* table, int64_t table_rows, void* y,
                      int64_t y_stride, int64_t T, int64_t H, int64_t D, int64_t R, int interleaved, void* stream) {
  clear_error();
  if (T < 0 || H < 0 || D < 0 || R < 0 || table_rows < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (R > D / 2) return fail(NIMBLE_ERR_SHAPE, "rotary: %lld pairs in heads of %lld", (long long)R, (long long)D);
  if (T > (1ll << 31) - 1 || H > (1 << 24) || D > (1 << 24) || H * D > (1ll << 31) - 1 || table_rows > (1ll << 31)) return fail(NIMBLE_ERR_ARG, "extent too large");
  if (x_stride < 0 || y_stride < 0 || (T > 1 && (x_stride < H * D || y_stride < H * D)))
    return fail(NIMBLE_ERR_ARG, "rotary: rows of %lld elements, %lld and %lld apart", (long long)(H * D), (long long)x_stride, (long long)y_stride);
  if (T == 0 || H == 0 || D == 0) return NIMBLE_OK;
  if (!x || !y || (R > 0 && (!positions || !table))) return fail(NIMBLE_ERR_NULL, "null tensor pointer");
  if (R > 0 && table_rows == 0) return fail(NIMBLE_ERR_SHAPE, "rotary: a table without positions");
  if (misaligned(x, 2) || misaligned(y, 2) || misaligned(positions, 8) || misaligned(table, 8))
    return fail(NIMBLE_ERR_ALIGN, "x and y must be 2-byte aligned, positions and table 8-byte");
  if (x == y && T > 1 && x_stride != y_stride) return fail(NIMBLE_ERR_ARG, "rotary: in place with two strides");
  const int rc = check_apart("rotary", {extent("y", y, T, H * D, y_stride)},
                             {extent("x", x == y ? nullptr : x, T, H * D, x_stride), extent("positions", R ? positions : nullptr, T * 8),
                              extent("the table", table, table_rows * R * 8)});
  if (rc != NIMBLE_OK) return rc;
  const RotaryArgs g{(const uint16_t*)x, (const long long*)positions, (const float2*)table, (uint16_t*)y, (long long)x_stride, (long long)y_stride,
                     (long long)table_rows, (long long)T, (int)H, (int)D, (int)R};
  const bool whole = D % 16 == 0 && R % 8 == 0 && !misaligned(x) && !misaligned(y) && !misaligned(table) && (T == 1 || (x_stride % 8 == 0 && y_stride % 8 == 0));
  auto launch = [&](auto kernel, int64_t threads) {
    hipLaunchKernelGGL(kernel, grid_of(threads, 256), dim3(256), 0, (hipStream_t)stream, g);
  };
  if (whole) {
    if (interleaved) launch(rotary_kernel<true>, T * H * (D / 16));
    else launch(rotary_kernel<false>, T * H * (D / 16));
  } else {
    if (interleaved) launch(rotary_any_kernel<true>, T * H * (D - R));
    else launch(rotary_any_kernel<false>, T * H * (D - R));
  }
  return check_hip_launch("rotary kernel launch");
}

int nimble_cache_write_dyn(const nimble_cache* cache, const nimble_sequences* seqs, const void* k, int64_t k_stride, const void* v,
                           int64_t v_stride, const void* q, int64_t q_stride, void* q_out, int64_t heads, const void* table,
                           int64_t table_rows, int64_t R, int interleaved, void* stream) {
  clear_error();
  int rc = check_cache(cache);
  if (rc == NIMBLE_OK) rc = check_sequences(seqs, cache->page);
  if (rc != NIMBLE_OK) return rc;
  const int64_t D = cache->D;
  if (table_rows < 0 || R < 0 || heads < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  if (table && (R % 8 || R > D / 2)) return fail(R > D / 2 ? NIMBLE_ERR_SHAPE : NIMBLE_ERR_ARG, "cache_write: %lld pairs in heads of %lld, a multiple of 8 needed", (long long)R, (long long)D);
  if (heads > 65536) return fail(NIMBLE_ERR_ARG, "extent too large");
  if (seqs->rows == 0 || seqs->count == 0) return NIMBLE_OK;
  rc = check_rows(k, k_stride, cache->kv_heads, D, "cache_write: k");
  if (rc == NIMBLE_OK) rc = check_rows(v, v_stride, cache->kv_heads, D, "cache_write: v");
  if (rc == NIMBLE_OK && q) rc = check_rows(q, q_stride, heads, D, "cache_write: q");
  if (rc != NIMBLE_OK) return rc;
  if (q && !q_out) return fail(NIMBLE_ERR_NULL, "null tensor pointer");
  if (q && q == q_out && q_stride != heads * D) return fail(NIMBLE_ERR_ARG, "cache_write: queries in place have to be contiguous");
  if (misaligned(q_out) || misaligned(table)) return fail(NIMBLE_ERR_ALIGN, "device pointers must be 16-byte aligned");
  if (table && R > 0 && table_rows == 0) return fail(NIMBLE_ERR_SHAPE, "cache_write: a table without positions");
  const auto [ck, cv, cks, cvs] = cache_extents(*cache);
  const auto [offsets, lengths, pages] = sequences_extents(*seqs);
  const int64_t T = seqs->rows, wide = heads * D, narrow = cache->kv_heads * D;
  rc = check_apart("cache_write", {extent("out", q ? q_out : nullptr, T, wide, wide), ck, cv, cks, cvs},
                   {extent("q", q == q_out ? nullptr : q, T, wide, q_stride), extent("k", k, T, narrow, k_stride),
                    extent("v", v, T, narrow, v_stride), extent("the table", table, (table_rows < 1ll << 40 ? table_rows : 1ll << 40) * R * 8), offsets, lengths, pages});
  if (rc == NIMBLE_OK && q == q_out)  // in place
    rc = check_apart("cache_write", {ck, cv, cks, cvs}, {extent("q", q, T, wide, q_stride)});
  if (rc != NIMBLE_OK) return rc;
  CacheWriteArgs g{};
  g.cache = cache_args(*cache);
  g.seqs = sequences_args(*seqs);
  g.k = (const uint16_t*)k;
  g.v = (const uint16_t*)v;
  g.q = (const uint16_t*)q;
  g.q_out = (uint16_t*)q_out;
  g.table = R > 0 ? (const float2*)table : nullptr;
  g.k_stride = k_stride;
  g.v_stride = v_stride;
  g.q_stride = q_stride;
  g.table_rows = table_rows;
  g.heads = (int)heads;
  g.R = g.table ? (int)R : 0;
  g.rows_each = rows_each(seqs->rows, 16);
  const bool int8 = cache->dtype == NIMBLE_I8;
  if (D == 64) {
    if (interleaved) launch_write<64, true>(g, int8, (hipStream_t)stream);
    else launch_write<64, false>(g, int8, (hipStream_t)stream);
  } else {
    if (interleaved) launch_write<128, true>(g, int8, (hipStream_t)stream);
    else launch_write<128, false>(g, int8, (hipStream_t)stream);
  }
  return check_hip_launch("cache write kernel launch");
}

int nimble_cache_read_dyn(const nimble_cache* cache, const nimble_sequences* seqs, void* k_out, void* v_out, int out_dtype, void* stream) {
  clear_error();
  int rc = check_cache(cache);
  if (rc == NIMBLE_OK) rc = check_sequences(seqs, cache->page);
  if (rc != NIMBLE_OK) return rc;
  if (out_dtype != NIMBLE_BF16 && out_dtype != NIMBLE_F32) return fail(NIMBLE_ERR_DTYPE, "unknown dtype %d", out_dtype);
  if (seqs->rows == 0 || seqs->count == 0) return NIMBLE_OK;
  if (!k_out || !v_out) return fail(NIMBLE_ERR_NULL, "null tensor pointer");
  if (misaligned(k_out) || misaligned(v_out)) return fail(NIMBLE_ERR_ALIGN, "device pointers must be 16-byte aligned");
  const auto [ck, cv, cks, cvs] = cache_extents(*cache);
  const auto [offsets, lengths, pages] = sequences_extents(*seqs);
  const int64_t bytes = seqs->rows * cache->kv_heads * cache->D * (out_dtype == NIMBLE_F32 ? 4 : 2);
  rc = check_apart("cache_read", {extent("k_out", k_out, bytes), extent("v_out", v_out, bytes)}, {ck, cv, cks, cvs, offsets, lengths, pages});
  if (rc != NIMBLE_OK) return rc;
  const CacheReadArgs g{cache_args(*cache), sequences_args(*seqs), k_out, v_out, rows_each(seqs->rows, 16)};
  if (cache->D == 64)
    launch_read<64>(g, cache->dtype == NIMBLE_I8, out_dtype == NIMBLE_F32, (hipStream_t)stream);
  else
    launch_read<128>(g, cache->dtype == NIMBLE_I8, out_dtype == NIMBLE_F32, (hipStream_t)stream);
  return check_hip_launch("cache read kernel launch");
}

}  // extern "C"
