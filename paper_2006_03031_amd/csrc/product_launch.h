// The launcher of a product's kernels; each file that includes this builds those of one type.
#ifndef NIMBLE_PRODUCT_LAUNCH_H_
#define NIMBLE_PRODUCT_LAUNCH_H_
#include <hip/hip_runtime.h>

#include "grouped_kernel.h"
#include "product_stream_kernel.h"
#include "product_tile_kernel.h"

namespace nimble {

static int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? NIMBLE_OK : fail(NIMBLE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

template <typename T, int GROUPS>
int launch_product(const ProductArgs& g, const nimble_product_plan& p, hipStream_t stream) {
  const unsigned tiles = (unsigned)p.tiles, tiles_n = (unsigned)((g.N + p.bn - 1) / p.bn);
  const dim3 grid(p.grid), block(p.block);
  if (p.kernel == NIMBLE_PRODUCT_TILES) {
    // tiles in flight are blocks of 8 rows of tiles.  Settled clocks, 8 rows / 4: 8 bits 16384 x 4096 x 4096 208 / 214 us, 8192 x 30528 x 1024
    // 294 / 297, 8192^3 388 / 384; bf16 16354 rows over 8 groups x 4096 x 1024 140 / 143, over 32 158 / 162.  2, 16 and 32 rows: 3 to 10 % longer
    // at 8192^3
    const int tiles_m = (int)(p.tiles / tiles_n), group_m = 8;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, g, tiles_m, (int)tiles_n, group_m); };
    auto pick = [&](auto f32) {
      constexpr bool F = decltype(f32)::value;
      switch (p.bm) {
        case 128: launch(product_tile_kernel<T, GROUPS, F, 128, 256, 3>); break;
        case 160: launch(product_tile_kernel<T, GROUPS, F, 160, 256, 2>); break;
        case 192: launch(product_tile_kernel<T, GROUPS, F, 192, 256, 2>); break;
        case 224: launch(product_tile_kernel<T, GROUPS, F, 224, 256, 2>); break;
        default: launch(product_tile_kernel<T, GROUPS, F, 256, 256, 2>); break;
      }
    };
    if (g.out_f32) pick(std::true_type{});
    else pick(std::false_type{});
    return launched("product tile kernel launch");
  }
  if (p.kernel == NIMBLE_PRODUCT_STREAM) {
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, g, tiles, tiles_n); };
    if (p.bm == 8) launch(product_stream_kernel<T, GROUPS, 1, 2, 4, kStreamStages, 8>);
    else if (p.bm == 16) launch(product_stream_kernel<T, GROUPS, 1, 2, 4, kStreamStages>);
    else if (p.bm == 32) launch(product_stream_kernel<T, GROUPS, 2, 2, 4, kStreamStages>);
    else if (p.k_waves == 4) launch(product_stream_kernel<T, GROUPS, 4, 4, 4, kStreamStages>);
    else launch(product_stream_kernel<T, GROUPS, 4, 4, 2, kStreamStages>);
    return launched("product stream kernel launch");
  }
  if (p.bm == 16)
    hipLaunchKernelGGL((product_direct_kernel<T, GROUPS, 1, 1, 8>), grid, block, 0, stream, g, tiles, tiles_n);
  else
    hipLaunchKernelGGL((product_direct_kernel<T, GROUPS, 4, 4, 4>), grid, block, 0, stream, g, tiles, tiles_n);
  return launched("product kernel launch");
}

}  // namespace nimble
#endif
