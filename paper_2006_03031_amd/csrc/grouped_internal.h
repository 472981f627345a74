// What the 8-bit and the grouped products share between host and device: arguments, plans, limits.
#ifndef NIMBLE_GROUPED_INTERNAL_H_
#define NIMBLE_GROUPED_INTERNAL_H_
#include "nimble_internal.h"

namespace nimble {

// y[r, n] = epi( sx[r] sw[e, n] sum_k x[r, k] w[e, n, k] + bias[e, n] ) for the rows r of each group e.  Rows of x and w are
// addressed in bytes: the kernels are the same for bf16 and for 8-bit integers up to the matrix instruction.
struct ProductArgs {
  const unsigned char* x;   // [rows, row_bytes]
  const unsigned char* w;   // [groups, N, row_bytes]
  const uint16_t* bias;        // [groups, N] or nullptr
  const float* x_scale;     // [rows]: 8-bit products only
  const float* w_scale;     // [groups, N]
  const long long* offsets; // [groups + 1], on the device; nullptr: one group of all rows
  void* y;                  // [rows, N]
  long long rows;
  int groups, N, row_bytes;
  int epilogue, out_f32;
};

// Groups whose first rows and tile counts a workgroup keeps in LDS (see GroupMap).
constexpr int kMostGroups = 1024;
constexpr int group_map_bytes(int most) { return most ? 2 * (most + 1) * 4 : 0; }
// LDS of a streaming workgroup: a ring of `stages` of 128 bytes of its rows and columns for each wave, scales and bias, the map of the groups.
constexpr int stream_lds_bytes(int rows, int columns, int k_waves, int stages, int groups) {
  return k_waves * stages * (rows + columns) * 128 + 3 * 64 * 4 + group_map_bytes(groups);
}
constexpr int kStreamStages = 2, kComputeUnitLds = 160 * 1024;
// A launch is of fewer than 2^32 threads; workgroups go round where there is more to do.
constexpr int64_t kMostWorkgroups = 1 << 21;
// 8-bit codes are down to -128: K * 128 * 128 stays below 2^31.
constexpr int64_t kMostK8 = 131071;
constexpr int64_t kMostK16 = 1ll << 22;

// Offsets inside a tile of 256 rows stay below 2^31.
constexpr int64_t kMostTileRowBytes = 1ll << 22, kMostTileColumns = 1ll << 20;

struct ProductShape {
  int64_t rows, groups, N, K;
  bool grouped, int8, out_f32;
  int64_t row_bytes() const { return int8 ? K : 2 * K; }
};

// The kernel, its tile and its grid for one call (integers of the host only: how the rows fall on the groups is not known here).
int plan_product(const ProductShape& s, nimble_product_plan* p);

}  // namespace nimble
#endif
