// The 8-bit and the grouped products where there are few rows: small tiles, K divided among the waves of a workgroup.
#ifndef NIMBLE_PRODUCT_STREAM_KERNEL_H_
#define NIMBLE_PRODUCT_STREAM_KERNEL_H_
#include "grouped_kernel.h"

namespace nimble {

// ---------------------------------------------------------------------------
// TM x TN blocks of 16 x 16 per workgroup; its KW waves take the stages of 128 bytes of K in turn and add their sums in LDS at the
// end.  Bound: the weights' bytes (one row block) or the chain of a workgroup's stages (few tiles).  A wave has a ring of S stages of its
// own, filled by its own loads of whole 128-byte lines, so that nothing in the loop waits for another wave.  (Fragments loaded
// from memory straight into registers ask for 16 lines per KiB eight times over, which bounds product_direct_kernel.)
//   Rows past the tile's last (x: of the group; w: of the weight) and pieces past the end of K are zeros that
// the buffer descriptors give, at no cost in memory traffic: a single row of x is read as one.
//   Bias and scales of the tile come to LDS with the first loads.
// ---------------------------------------------------------------------------
template <typename T, int GROUPS, int TM, int TN, int KW, int S, int XR = 16 * TM>
__global__ void __launch_bounds__(KW * 64) product_stream_kernel(ProductArgs g, unsigned tiles, unsigned tiles_n) {
  constexpr int BM = 16 * TM, BN = 16 * TN;
  constexpr int XL = XR / 8, LD = XL + 2 * TN;      // loads of 8 rows per stage
  constexpr int SLOT = (XR + BN) * 8;               // uint4
  constexpr int RING = S * SLOT;
  static_assert(S * LD <= 60, "the wait counter holds 63");
  static_assert(XR == 16 * TM || (TM == 1 && XR == 8), "x rows");
  static_assert(RING >= TM * TN * 64, "a wave's sums go where its ring was");
  typedef typename T::Acc Acc;
  __shared__ __attribute__((aligned(16))) uint4 smem[KW][RING];
  __shared__ __attribute__((aligned(16))) float values[3][64];  // scales of rows and columns, bias
  __shared__ GroupMap<GROUPS> map;
  static_assert(sizeof(smem) + sizeof(values) + group_map_bytes(GROUPS) == stream_lds_bytes(XR, BN, KW, S, GROUPS), "LDS as the host takes it");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (GROUPS) {
    map_groups<XR>(g, map);
    __syncthreads();
  }
  const int KS = (g.row_bytes + 127) >> 7, left = g.row_bytes - (KS - 1) * 128;
  const int ld_row = lane >> 3, fr_row = lane & 15, fr_q = lane >> 4;
  const bool parked = (g.N & 1) == 0;  // (odd N: pairs of columns start anywhere)
  // chunk c of row r lies at c ^ ((r >> 1) & 7); the two loads of 16 rows differ in it
  const int ld_c[2] = {(lane & 7) ^ (ld_row >> 1), (lane & 7) ^ (4 + (ld_row >> 1))};
  const int fr_phys = fr_q ^ ((fr_row >> 1) & 7), half = (fr_phys ^ 4) - fr_phys;
  // (8 rows of x: the matrix instruction's other 8 rows take them again, for results that nobody asks for)
  const int x_row = XR == 8 ? fr_row & 7 : fr_row, x_phys = fr_q ^ ((x_row >> 1) & 7), x_half = (x_phys ^ 4) - x_phys, x_at = x_row * 8 + x_phys;
  const uint4* ring = smem[wave];
  const uint32_t ring_lds = __builtin_amdgcn_readfirstlane(lds_addr_of(ring));
  uint32_t off[LD];
#pragma unroll
  for (int u = 0; u < LD; ++u) {
    const int row = (u < XL ? 8 * u : 8 * (u - XL)) + ld_row;
    off[u] = (uint32_t)(row * g.row_bytes + ld_c[(u < XL ? u : u - XL) & 1] * 16);
  }
  const uint32_t past[2] = {ld_c[0] * 16 >= left ? 0x80000000u : 0u, ld_c[1] * 16 >= left ? 0x80000000u : 0u};
  for (unsigned b = blockIdx.x; b < tiles; b += gridDim.x) {
    ProductTile tile;
    const unsigned t = b / tiles_n;
    if (!find_tile<XR, BN>(g, map, (int)t, (int)(b - t * tiles_n), tile)) return;
    const int columns = min(BN, g.N - tile.n0);
    const long long c0 = (long long)tile.group * g.N + tile.n0;
    const rsrc_t xr = descriptor(g.x + (long long)tile.row0 * g.row_bytes, (uint32_t)tile.rows * (uint32_t)g.row_bytes);
    const rsrc_t wr = descriptor(g.w + c0 * g.row_bytes, (uint32_t)columns * (uint32_t)g.row_bytes);
    auto load = [&](int ks, int slot) {
      const bool real = ks < KS;
      const uint32_t end = ks == KS - 1 ? 0xffffffffu : 0u;
      rsrc_t x = xr, w = wr;
      x[2] = real ? x[2] : 0;
      w[2] = real ? w[2] : 0;
#pragma unroll
      for (int u = 0; u < LD; ++u)
        dma16_buffer(off[u] | (past[(u < XL ? u : u - XL) & 1] & end), u < XL ? x : w, (uint32_t)(real ? ks : 0) * 128u, ring_lds + slot * SLOT * 16 + u * 1024);
    };
    if (wave == 0) {
      if (T::kInt8) {
        dma4_buffer(lane * 4u, descriptor(g.x_scale + tile.row0, (uint32_t)tile.rows * 4u), __builtin_amdgcn_readfirstlane(lds_addr_of(values[0])));
        dma4_buffer(lane * 4u, descriptor(g.w_scale + c0, (uint32_t)columns * 4u), __builtin_amdgcn_readfirstlane(lds_addr_of(values[1])));
      }
      if (g.epilogue != NIMBLE_EPI_NONE && parked)
        dma4_buffer(lane * 4u, descriptor(g.bias + c0, (uint32_t)columns * 2u), __builtin_amdgcn_readfirstlane(lds_addr_of(values[2])));
    }
#pragma unroll
    for (int s = 0; s < S; ++s) load(wave + s * KW, s);
    Acc acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = Acc{0, 0, 0, 0};
    int slot = 0;
    for (int ks = wave; ks < KS; ks += KW) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 1) * LD) : "memory");
      const uint4 *rw = ring + slot * SLOT + (XR + fr_row) * 8 + fr_phys, *rx = ring + slot * SLOT + x_at;
      uint4 x[TM][2], w[TN][2];
#pragma unroll
      for (int i = 0; i < TN; ++i) w[i][0] = rw[16 * i * 8], w[i][1] = rw[16 * i * 8 + half];
#pragma unroll
      for (int j = 0; j < TM; ++j) x[j][0] = rx[16 * j * 8], x[j][1] = rx[16 * j * 8 + x_half];
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      load(ks + S * KW, slot);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j) acc[i][j] = T::mfma(w[i][h], x[j][h], acc[i][j]);
      slot = slot + 1 == S ? 0 : slot + 1;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the loads past the end write zeros)
    Acc* sums = (Acc*)smem[wave];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) sums[(i * TM + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < TM * TN * 64; o += KW * 64) {
      Acc s = ((const Acc*)smem[0])[o];
#pragma unroll
      for (int k = 1; k < KW; ++k) s += ((const Acc*)smem[k])[o];
      const int l = o & 63, block = o >> 6, i = block / TM, j = block % TM;
      const int r = 16 * j + (l & 15), c = 16 * i + 4 * (l >> 4);
      if (r >= tile.rows || c >= columns) continue;
      float v[4], bias[4] = {0.f, 0.f, 0.f, 0.f};
      if (g.epilogue != NIMBLE_EPI_NONE) {
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = bf2f(parked ? ((const u16*)values[2])[c + e] : g.bias[c0 + min(c + e, columns - 1)]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = T::kInt8 ? fmaf((float)s[e], values[0][r] * values[1][c + e], bias[e]) : (float)s[e] + bias[e];
      store4(g, v, (long long)tile.row0 + r, tile.n0 + c);
    }
    __syncthreads();  // (the next tile's loads come where the sums are)
  }
}

}  // namespace nimble
#endif
