// Device entry points and launchers of the 8-bit and the grouped products.
//   quantize_kernel.h        quantize_rows_kernel: rows to 8-bit codes and a scale each.
//   grouped_kernel.h         the map from workgroups to the tiles of groups that only the device knows, loads through buffer descriptors,
//       and product_direct_kernel: operands of any alignment.
//   product_stream_kernel.h  product_stream_kernel: small tiles, K divided among a workgroup's waves.
//   product_tile_kernel.h    product_tile_kernel: large tiles by four waves, the first stages of a tile loaded during the last ones of the tile before.
#include <hip/hip_runtime.h>

#include "grouped_internal.h"
#include "grouped_kernel.h"
#include "quantize_kernel.h"

namespace nimble {

static int check_hip(hipError_t e, const char* what) {
  if (e == hipSuccess) return NIMBLE_OK;
  return fail(NIMBLE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}
static bool misaligned(const void* p, unsigned to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

// (product_launch.h; built in product_bf16_grouped.hip, product_i8_grouped.hip and product_i8.hip)
template <typename T, int GROUPS>
int launch_product(const ProductArgs& g, const nimble_product_plan& p, hipStream_t stream);

// What the three products have in common behind their checks of types and extents.
static int run_product(ProductArgs g, int64_t R, int64_t E, int64_t N, int64_t K, bool grouped, bool int8, hipStream_t stream) {
  if (g.epilogue < NIMBLE_EPI_NONE || g.epilogue > NIMBLE_EPI_BIAS_GELU_ERF) return fail(NIMBLE_ERR_ARG, "unknown epilogue %d", g.epilogue);
  if (grouped && E < 0) return fail(NIMBLE_ERR_ARG, "negative extent");
  nimble_product_plan p;
  int rc = nimble_product_plan_of(R, grouped ? E : -1, N, K, int8 ? NIMBLE_I8 : NIMBLE_BF16, g.out_f32, &p);
  if (rc != NIMBLE_OK) return rc;
  if (R == 0 || N == 0 || (grouped && E == 0)) return NIMBLE_OK;
  if (!g.y || (grouped && !g.offsets) || (int8 && (!g.x_scale || !g.w_scale)) || (K > 0 && (!g.x || !g.w)) ||
      (g.epilogue != NIMBLE_EPI_NONE && !g.bias))
    return fail(NIMBLE_ERR_NULL, "null tensor pointer");
  if (misaligned(g.x) || misaligned(g.w) || misaligned(g.y) || misaligned(g.x_scale) || misaligned(g.w_scale) || misaligned(g.bias))
    return fail(NIMBLE_ERR_ALIGN, "device pointers must be 16-byte aligned");
  if (misaligned(g.offsets, 8)) return fail(NIMBLE_ERR_ALIGN, "offsets must be 8-byte aligned");
  g.rows = R;
  g.groups = grouped ? (int)E : 1;
  g.N = (int)N;
  g.row_bytes = (int)(int8 ? K : 2 * K);
  if (g.epilogue == NIMBLE_EPI_NONE) g.bias = nullptr;
  if (!int8) return launch_product<OfBf16, kMostGroups>(g, p, stream);
  return grouped ? launch_product<OfInt8, kMostGroups>(g, p, stream) : launch_product<OfInt8, 0>(g, p, stream);
}

}  // namespace nimble

using namespace nimble;

extern "C" {

int nimble_quantize_rows_dyn(const void* x, int x_dtype, void* q, void* scale, int64_t rows, int64_t K, int64_t cols, void* stream) {
  clear_error();
  const int64_t shape[2] = {rows, K};
  int64_t q_shape[2], scale_shape[1];
  if (x_dtype != NIMBLE_BF16 && x_dtype != NIMBLE_F32) return fail(NIMBLE_ERR_DTYPE, "unknown dtype %d", x_dtype);
  const int rc = nimble_quantize_rows_shape(shape, 2, cols, q_shape, scale_shape);
  if (rc != NIMBLE_OK) return rc;
  if (rows > (1ll << 31) - 1) return fail(NIMBLE_ERR_ARG, "extent too large");
  if (rows == 0) return NIMBLE_OK;
  if ((K > 0 && !x) || (q_shape[1] > 0 && !q) || !scale) return fail(NIMBLE_ERR_NULL, "null tensor pointer");
  if (misaligned(x) || misaligned(q) || misaligned(scale)) return fail(NIMBLE_ERR_ALIGN, "device pointers must be 16-byte aligned");
  const QuantizeArgs g{x, (signed char*)q, (float*)scale, (long long)rows, (int)K, (int)q_shape[1]};
  // A wave per row where there are rows enough for every SIMD and a row is at most two groups per lane, else four: 8177 rows of 4096 as calls in
  // a row, with eight groups per lane of one wave 27.1 us (120 registers), with two of four waves 24.0.
  const bool wave = rows >= 2048 && K <= 1024;
  const int64_t groups = wave ? (rows + 3) / 4 : rows;
  const dim3 grid((unsigned)(groups < kMostWorkgroups ? groups : kMostWorkgroups)), block(256);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, (hipStream_t)stream, g); };
  if (x_dtype == NIMBLE_F32) {
    if (wave) launch(quantize_rows_kernel<true, 1, 2>);
    else if (K <= 4096) launch(quantize_rows_kernel<true, 4, 2>);
    else if (K <= 8192) launch(quantize_rows_kernel<true, 4, 4>);
    else launch(quantize_rows_kernel<true, 4, 8>);
  } else {
    if (wave) launch(quantize_rows_kernel<false, 1, 2>);
    else if (K <= 4096) launch(quantize_rows_kernel<false, 4, 2>);
    else if (K <= 8192) launch(quantize_rows_kernel<false, 4, 4>);
    else launch(quantize_rows_kernel<false, 4, 8>);
  }
  return check_hip(hipGetLastError(), "quantize kernel launch");
}

int nimble_dense_i8_dyn(const void* x, const void* x_scale, const void* w, const void* w_scale, const void* bias, void* y, int64_t M,
                        int64_t N, int64_t K, int epilogue, int out_dtype, void* stream) {
  clear_error();
  ProductArgs g{};
  g.x = (const unsigned char*)x;
  g.w = (const unsigned char*)w;
  g.bias = (const uint16_t*)bias;
  g.x_scale = (const float*)x_scale;
  g.w_scale = (const float*)w_scale;
  g.y = y;
  g.epilogue = epilogue;
  g.out_f32 = out_dtype;
  return run_product(g, M, 1, N, K, false, true, (hipStream_t)stream);
}

int nimble_grouped_dense_dyn(const void* x, const void* w, const void* bias, const void* offsets, void* y, int64_t R, int64_t E,
                             int64_t N, int64_t K, int epilogue, int out_dtype, void* stream) {
  clear_error();
  ProductArgs g{};
  g.x = (const unsigned char*)x;
  g.w = (const unsigned char*)w;
  g.bias = (const uint16_t*)bias;
  g.offsets = (const long long*)offsets;
  g.y = y;
  g.epilogue = epilogue;
  g.out_f32 = out_dtype;
  return run_product(g, R, E, N, K, true, false, (hipStream_t)stream);
}

int nimble_grouped_dense_i8_dyn(const void* x, const void* x_scale, const void* w, const void* w_scale, const void* bias,
                                const void* offsets, void* y, int64_t R, int64_t E, int64_t N, int64_t K, int epilogue, int out_dtype,
                                void* stream) {
  clear_error();
  ProductArgs g{};
  g.x = (const unsigned char*)x;
  g.w = (const unsigned char*)w;
  g.bias = (const uint16_t*)bias;
  g.x_scale = (const float*)x_scale;
  g.w_scale = (const float*)w_scale;
  g.offsets = (const long long*)offsets;
  g.y = y;
  g.epilogue = epilogue;
  g.out_f32 = out_dtype;
  return run_product(g, R, E, N, K, true, true, (hipStream_t)stream);
}

}  // extern "C"
