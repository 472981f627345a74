// The 8-bit and the grouped products in large tiles by four waves.
#ifndef NIMBLE_PRODUCT_TILE_KERNEL_H_
#define NIMBLE_PRODUCT_TILE_KERNEL_H_
#include "grouped_kernel.h"

namespace nimble {

// ---------------------------------------------------------------------------
// Tiles of BM x BN by four waves in two rows and two columns, one wave per SIMD, one tile after the other: a ring of S stages
// of 128 bytes of K in LDS, each stage multiplied in four quarters, the fragments that the next quarter needs read and the
// stage S ahead loaded in between its MFMAs (the schedule of gemm_quarter_kernel.h).  A stage of 128 bytes takes the matrix cores the
// same time in either type: 64 k of bf16, 128 k of int8.  Bound: MFMA and, with real data, the power that products, fragment reads and
// loads take together; with short K also the ends of the tiles.
//   Columns go to the matrix instruction's rows such that a lane holds eight neighbouring ones of bf16 (four of f32): 16 bytes, 64
// contiguous ones with its three neighbours, stored from registers as they are.  The swizzle of the weights' rows in LDS
// follows (see b_swizzle).  With the outputs brought into whole lines through LDS first, 8192 x 4096 x 1024 in 8 bits took 53.6 us, stored from
// registers 36.4.
//   The loads past a tile's last stage are the next tile's first ones, and the stores of a tile's end stay in flight while the next
// begins.  To put a tile's sums aside and finish them in between the next tile's products as well (128 x 256, twice 128 registers
// of sums) gained nothing: 41.3 us, with it 40.3; one wave issues an instruction in four clocks at most, and products, reads and
// loads leave it few.
//   Loads go through buffer descriptors that end with the tile's last row (of its group, of the weight): rows past it, which
// belong to another group or to nobody, come back as zeros, and so does, by an offset past every descriptor, what lies behind
// the end of K in the last stage.  Stores past the last row or column are dropped in the same way.  So every tile runs the same code
// whatever its number of rows.
//   Tiles are told from the offsets of the groups (GroupMap), which the workgroup reads once.
//   Measured with settled clocks, 8 bits / bf16: 8192^3 394 / 820 us (2790 / 1340 T); 8192 x 4096 x 1024 with bias 34.3-35.1 / 61.4-63.6, with GELU
// to bf16 42.7-45.5 / 69-74 (half of 16384 rows), to f32 47.7-50.4: the spread is that of two cards.
// ---------------------------------------------------------------------------
#define NIMBLE_INLINE __attribute__((always_inline))
template <int N>
using Int = std::integral_constant<int, N>;
// f(Int<FROM>{}), f(Int<FROM + 1>{}), ... up to TO: indexes that are constants for the compiler from the start, since
// the sums have to stay in registers that they name.
template <int FROM, int TO, typename F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (FROM < TO) {
    f(Int<FROM>{});
    each<FROM + 1, TO>(f);
  }
}
// 16 bytes per lane to the descriptor's byte voff + soff, through the L2 (see store_through); past its end nothing.
__device__ __forceinline__ void store16_buffer(uint4 v, uint32_t voff, rsrc_t rsrc, uint32_t soff) {
  asm volatile("buffer_store_dwordx4 %0, %1, %2, %3 offen sc1\n\ts_nop 1" ::"v"(__builtin_bit_cast(i32x4, v)), "v"(voff),
               "s"(rsrc), "s"(soff)
               : "memory");
}

// The matrix instruction as a volatile statement (see mfma_acc): C is the sum or, for a tile's first, zero; with a load
// behind it; with the wait states that let the sums be read (`last`).
#define NIMBLE_PRODUCT_MFMA(T, INSN)                                                                                          \
  template <bool ZERO>                                                                                                        \
  __device__ __forceinline__ void mfma_in_place(T::Acc& acc, const uint4& a, const uint4& b) {                                \
    if (ZERO)                                                                                                                 \
      asm volatile(INSN " %0, %1, %2, 0" : "+a"(acc) : "v"(__builtin_bit_cast(i32x4, a)), "v"(__builtin_bit_cast(i32x4, b))); \
    else                                                                                                                      \
      asm volatile(INSN " %0, %1, %2, %0" : "+a"(acc) : "v"(__builtin_bit_cast(i32x4, a)), "v"(__builtin_bit_cast(i32x4, b))); \
  }                                                                                                                           \
  __device__ __forceinline__ void mfma_in_place_last(T::Acc& acc, const uint4& a, const uint4& b, int last) {                 \
    asm volatile(INSN                                                                                                         \
                 " %0, %1, %2, %0\n\t"                                                                                        \
                 "s_cmp_eq_u32 %3, 0\n\t"                                                                                     \
                 "s_cbranch_scc1 .Lnimble_product_done_%=\n\t"                                                                \
                 "s_nop 15\n\t"                                                                                               \
                 "s_nop 15\n"                                                                                                 \
                 ".Lnimble_product_done_%=:"                                                                                  \
                 : "+a"(acc)                                                                                                  \
                 : "v"(__builtin_bit_cast(i32x4, a)), "v"(__builtin_bit_cast(i32x4, b)),                                      \
                   "s"(__builtin_amdgcn_readfirstlane(last))                                                                  \
                 : "scc");                                                                                                    \
  }                                                                                                                           \
  template <bool ZERO>                                                                                                        \
  __device__ __forceinline__ void mfma_in_place_load(T::Acc& acc, const uint4& a, const uint4& b, uint32_t voff, rsrc_t rsrc,  \
                                                     uint32_t soff, uint32_t lds_base, uint32_t lds_off) {                    \
    if (ZERO)                                                                                                                 \
      asm volatile("s_add_u32 m0, %6, %7\n\t" INSN                                                                            \
                   " %0, %1, %2, 0\n\t"                                                                                       \
                   "buffer_load_dwordx4 %3, %4, %5 offen lds"                                                                 \
                   : "+a"(acc)                                                                                                \
                   : "v"(__builtin_bit_cast(i32x4, a)), "v"(__builtin_bit_cast(i32x4, b)), "v"(voff), "s"(rsrc), "s"(soff),   \
                     "s"(lds_base), "s"(lds_off)                                                                              \
                   : "memory", "m0", "scc");                                                                                  \
    else                                                                                                                      \
      asm volatile("s_add_u32 m0, %6, %7\n\t" INSN                                                                            \
                   " %0, %1, %2, %0\n\t"                                                                                      \
                   "buffer_load_dwordx4 %3, %4, %5 offen lds"                                                                 \
                   : "+a"(acc)                                                                                                \
                   : "v"(__builtin_bit_cast(i32x4, a)), "v"(__builtin_bit_cast(i32x4, b)), "v"(voff), "s"(rsrc), "s"(soff),   \
                     "s"(lds_base), "s"(lds_off)                                                                              \
                   : "memory", "m0", "scc");                                                                                  \
  }
NIMBLE_PRODUCT_MFMA(OfBf16, "v_mfma_f32_16x16x32_bf16")
NIMBLE_PRODUCT_MFMA(OfInt8, "v_mfma_i32_16x16x64_i8")
#undef NIMBLE_PRODUCT_MFMA

// A sum out of its accumulation register, where the source has it: left to itself the compiler fetches all sums of a tile before it
// needs them, and spills.
template <typename V>
__device__ __forceinline__ V read_sum(const V& sum) {
  V v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(sum));
  return v;
}

// Bias (bf16), column scales and row scales of a tile, in LDS.
template <int BM, int BN>
struct TileValues {
  float w_scale[BN], x_scale[(BM + 63) / 64 * 64];  // (they come in pieces of 64)
  u16 bias[BN];
};
template <int BM, int BN, int S>
constexpr int kProductTileBytes = S * (BM + BN) * 128 + 2 * (int)sizeof(TileValues<BM, BN>);

template <typename T, int GROUPS, bool OUT_F32, int BM, int BN, int S>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1)))
    product_tile_kernel(ProductArgs g, int tiles_m, int tiles_n, int group_m) {
  constexpr int WM = BM / 2, WN = BN / 2;
  constexpr int TM = WM / 16, TN = WN / 16;
  constexpr int H0 = (TM + 1) / 2, H1 = TM - H0;  // 16-row tiles in the two halves of a wave's rows
  constexpr int G = TN / 2;                       // 16-column tiles in either half of its columns
  static_assert(BM % 32 == 0 && H1 >= 1 && BN % 128 == 0, "whole 16 x 16 tiles in either half of a wave's rows and columns");
  static_assert(kProductTileBytes<BM, BN, S> + (GROUPS ? (int)sizeof(GroupMap<GROUPS>) : 0) <= 160 * 1024, "LDS");
  constexpr int SLOT = (BM + BN) * 128;  // bytes
  constexpr int LDT = TM + TN;           // loads per wave and stage: H0, G, G, H1 of 32 rows each
  constexpr int FLIGHT = (S - 1) * LDT;  // loads that may be in flight at a barrier
  static_assert(FLIGHT + G + H1 <= 63, "the wait counter holds 63");
  constexpr int MFMAS = 2 * TM * TN;     // of a stage
  constexpr int STORES = TM * TN / 2 * (OUT_F32 ? 2 : 1);  // per wave, of a tile's end
  constexpr int OS = OUT_F32 ? 4 : 2;
  typedef TileValues<BM, BN> Values;
  typedef typename T::Acc Acc;
  __shared__ __attribute__((aligned(16))) unsigned char smem[kProductTileBytes<BM, BN, S>];
  __shared__ GroupMap<GROUPS> map;
  if (GROUPS) {
    map_groups<BM>(g, map);
    __syncthreads();
    tiles_m = __builtin_amdgcn_readfirstlane(map.ends[g.groups - 1]);
  }
  const int tiles_total = tiles_m * tiles_n;
  if ((int)blockIdx.x >= tiles_total) return;
  auto tile_at = [&](int t, ProductTile& tile) {
    int tm, tn;
    tile_of_block(t, tiles_total, tiles_m, tiles_n, group_m, tm, tn);
    find_tile<BM, BN>(g, map, tm, tn, tile);
  };

  // Stages of a tile: as many at least as are loaded ahead, those past the end of K of zeros.  `tight`: the pieces past the end of K lie
  // in these first stages.
  int KS = __builtin_amdgcn_readfirstlane(max((g.row_bytes + 127) >> 7, S));
  asm volatile("" : "+s"(KS));  // (the compiler, once it knows that S stages follow each other, spills)
  const bool tight = KS == S && g.row_bytes < S * 128;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  // row of the tile behind row q of half h of A (the halves of both rows of waves), the same for B
  auto a_row = [](int h, int q) {
    const int n = 16 * (h ? H1 : H0);
    return h * 16 * H0 + (q >= n ? WM - n : 0) + q;
  };
  auto b_row = [](int h, int q) { return h * 16 * G + (q >= 16 * G ? WN - 16 * G : 0) + q; };
  // Chunk c of row r lies at c ^ swizzle(r).  A fragment read takes 16 rows and is free of bank conflicts where each value of
  // the swizzle comes twice: of A, and of B for f32, 16 rows in a row; of B for bf16 rows 8 a + 4 x + b of 32, a, b < 4.
  auto a_swizzle = [](int r) { return (r >> 1) & 7; };
  auto b_swizzle = [](int r) { return OUT_F32 ? (r >> 1) & 7 : ((r >> 1) & 1) | ((r >> 2) & 6); };
  // loads of a stage in the order in which they are needed: H0 of A, G of B, G of B, H1 of A.  Offset of the lane, and
  // where in a slot the wave's 8 rows go.
  const int ld_row = tid >> 3;
  const int ld_a = (tid & 7) ^ a_swizzle(ld_row), ld_b = (tid & 7) ^ b_swizzle(ld_row);  // (the passes are 32 rows apart)
  uint32_t off[LDT], lds_off[LDT];
  auto of_a = [](int u) { return u < H0 || u >= H0 + TN; };
  auto row_of = [&](int u, int q) {
    const int h = of_a(u) ? u >= H0 : u >= H0 + G, base = of_a(u) ? (h ? u - TN - H0 : u) * 32 : (u - H0 - G * h) * 32;
    return of_a(u) ? a_row(h, base + q) : b_row(h, base + q);
  };
  // for the loads of a stage: pieces past the end of K are asked for past the end of the descriptor.  (The lane's row goes through an
  // empty statement: else the compiler keeps the addresses of every place that sets them alive beside each other, and spills.)
  auto set_off = [&](int stage) {
    int row = ld_row;
    asm volatile("" : "+v"(row));
    const int left = g.row_bytes - stage * 128;
#pragma unroll
    for (int u = 0; u < LDT; ++u) {
      const int c = (of_a(u) ? ld_a : ld_b) * 16;
      off[u] = c < left ? (uint32_t)(row_of(u, row) * g.row_bytes + c) : 0x80000000u;
    }
  };
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr_of(smem));
#pragma unroll
  for (int u = 0; u < LDT; ++u) lds_off[u] = (of_a(u) ? 0 : BM * 128) + row_of(u, wave * 8) * 128;
  set_off(0);
  auto a_desc = [&](const ProductTile& t) {
    return descriptor(g.x + (long long)t.row0 * g.row_bytes, (uint32_t)t.rows * (uint32_t)g.row_bytes);
  };
  auto b_desc = [&](const ProductTile& t) {
    return descriptor(g.w + ((long long)t.group * g.N + t.n0) * g.row_bytes, (uint32_t)min(BN, g.N - t.n0) * (uint32_t)g.row_bytes);
  };
  rsrc_t a_src, b_src;
  uint32_t at = 0;
  auto src = [&](int u) NIMBLE_INLINE { return of_a(u) ? a_src : b_src; };

  const int fr_row = lane & 15, fr_q = lane >> 4;
  // row of B that is row r of the matrix instruction's tile i
  auto b_tile_row = [](int i, int r) { return OUT_F32 ? 16 * i + r : 32 * (i >> 1) + 8 * (r >> 2) + 4 * (i & 1) + (r & 3); };
  const int a_phys = fr_q ^ a_swizzle(fr_row), b_phys = fr_q ^ b_swizzle(b_tile_row(0, fr_row));
  const int a_half = (a_phys ^ 4) - a_phys, b_half = (b_phys ^ 4) - b_phys;
  const uint4* a_rd = (const uint4*)smem + (wm * WM + fr_row) * 8 + a_phys;
  const uint4* b_rd = (const uint4*)smem + (BM + wn * WN + b_tile_row(0, fr_row)) * 8 + b_phys;
  // rows of tile i behind those of tile 0 (the swizzle is the same: whole 16 rows, or 4 of which it does not depend on bit 2)
  auto b_step = [](int i) { return (OUT_F32 ? 16 * i : 32 * (i >> 1) + 4 * (i & 1)) * 8; };

  Acc acc[TN][TM];

  Values* const values = (Values*)(smem + S * SLOT);
  // 4 bytes per lane; past the end of the row or of the tile's rows nothing is needed, and zeros come
  auto fetch_values = [&](const ProductTile& t, const Values* to) {
    const long long c0 = (long long)t.group * g.N + t.n0;
    const int columns = min(BN, g.N - t.n0);
    if (g.epilogue != NIMBLE_EPI_NONE && wave < BN / 128)
      dma4_buffer((uint32_t)(wave * 256 + lane * 4), descriptor((const u16*)g.bias + c0, (uint32_t)columns * 2u),
                  __builtin_amdgcn_readfirstlane(lds_addr_of(to->bias)) + wave * 256);
    if (T::kInt8) {
      if (wave < BN / 64)
        dma4_buffer((uint32_t)(wave * 256 + lane * 4), descriptor(g.w_scale + c0, (uint32_t)columns * 4u),
                    __builtin_amdgcn_readfirstlane(lds_addr_of(to->w_scale)) + wave * 256);
      if (wave < (BM + 63) / 64)
        dma4_buffer((uint32_t)(wave * 256 + lane * 4), descriptor(g.x_scale + t.row0, (uint32_t)t.rows * 4u),
                    __builtin_amdgcn_readfirstlane(lds_addr_of(to->x_scale)) + wave * 256);
    }
  };

  // The end of a tile, in blocks of two 16-column tiles 2 p, 2 p + 1 and 16 rows j.  A lane's eight values are columns 8 fr_q .. + 7 of
  // the 32 (bf16), or 4 fr_q .. + 3 of either 16 (f32), of row fr_row.
  const uint32_t out_row = (uint32_t)g.N * OS * 16;   // 16 rows
  const int out_col = OUT_F32 ? 4 * fr_q : 8 * fr_q;  // first column of a lane within its 32
  const uint32_t out_off = (uint32_t)((wm * WM + fr_row) * g.N + wn * WN + out_col) * OS;
  auto column = [&](int p, int k) { return wn * WN + 32 * p + out_col + (OUT_F32 ? 16 * (k >> 2) + (k & 3) : k); };
  auto finish = [&](const ProductTile& t, const Values& val, auto gelu) NIMBLE_INLINE {
    const rsrc_t out = descriptor((unsigned char*)g.y + ((long long)t.row0 * g.N + t.n0) * OS,
                                  (uint32_t)((t.rows - 1) * g.N + min(BN, g.N - t.n0)) * OS);
    float xs[TM];
#pragma unroll
    for (int j = 0; j < TM; ++j) xs[j] = T::kInt8 ? val.x_scale[wm * WM + j * 16 + fr_row] : 1.0f;
    each<0, TN / 2>([&](auto p_tag) NIMBLE_INLINE {
      constexpr int p = decltype(p_tag)::value;
      float ws[8], bs[8];
#pragma unroll
      for (int k = 0; k < 8; k += 4) {
        const int c = column(p, k);
        const float4 w4 = T::kInt8 ? *(const float4*)(val.w_scale + c) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
        const uint2 bb = g.epilogue != NIMBLE_EPI_NONE ? *(const uint2*)(val.bias + c) : make_uint2(0, 0);
        ws[k] = w4.x, ws[k + 1] = w4.y, ws[k + 2] = w4.z, ws[k + 3] = w4.w;
        bs[k] = bf2f((u16)(bb.x & 0xffff)), bs[k + 1] = bf2f((u16)(bb.x >> 16));
        bs[k + 2] = bf2f((u16)(bb.y & 0xffff)), bs[k + 3] = bf2f((u16)(bb.y >> 16));
      }
      const uint32_t c = (uint32_t)(t.n0 + wn * WN + 32 * p + out_col);
      each<0, TM>([&](auto j_tag) NIMBLE_INLINE {
        constexpr int j = decltype(j_tag)::value;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const auto held = acc[2 * p + (k >> 2)][j][k & 3];
          const float sum = (float)read_sum(held);
          v[k] = T::kInt8 ? fmaf(sum, xs[j] * ws[k], bs[k]) : sum + bs[k];
        }
        if constexpr (decltype(gelu)::value) gelu_of<OUT_F32>(v);
        if constexpr (OUT_F32) {
#pragma unroll
          for (int x = 0; x < 2; ++x)
            store16_buffer(__builtin_bit_cast(uint4, make_float4(v[4 * x], v[4 * x + 1], v[4 * x + 2], v[4 * x + 3])),
                           c + 16 * x < (uint32_t)g.N ? out_off + (32 * p + 16 * x) * OS : 0x80000000u, out, j * out_row);
        } else {
          store16_buffer(make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])),
                         c < (uint32_t)g.N ? out_off + 32 * p * OS : 0x80000000u, out, j * out_row);
        }
      });
    });
  };

  // ---- the walk
  ProductTile tile, next_tile;
  tile_at(blockIdx.x, tile);
  a_src = a_desc(tile);
  b_src = b_desc(tile);
  fetch_values(tile, values);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    if (tight) set_off(s);
#pragma unroll
    for (int u = 0; u < LDT; ++u) dma16_buffer(off[u], src(u), s * 128, lds0 + s * SLOT + lds_off[u]);
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(FLIGHT + G + H1) : "memory");
  __syncthreads();

  uint4 xa0[H0][2], xa1[H1][2], wb0[G][2], wb1[G][2];  // [tile][k half]
  auto rd_a0 = [&](int s, int x) NIMBLE_INLINE { xa0[x % H0][x / H0] = a_rd[s * (SLOT / 16) + (x % H0) * 128 + (x / H0) * a_half]; };
  auto rd_a1 = [&](int s, int x) NIMBLE_INLINE { xa1[x % H1][x / H1] = a_rd[s * (SLOT / 16) + (H0 + x % H1) * 128 + (x / H1) * a_half]; };
  auto rd_b0 = [&](int s, int x) NIMBLE_INLINE { wb0[x % G][x / G] = b_rd[s * (SLOT / 16) + b_step(x % G) + (x / G) * b_half]; };
  auto rd_b1 = [&](int s, int x) NIMBLE_INLINE { wb1[x % G][x / G] = b_rd[s * (SLOT / 16) + b_step(G + x % G) + (x / G) * b_half]; };
#pragma unroll
  for (int x = 0; x < 2 * H0; ++x) rd_a0(0, x);
#pragma unroll
  for (int x = 0; x < TN; ++x) rd_b0(0, x);

  // S - 1 whole stages may be in flight; with `lax` also the stores of the tile before, all of them behind the loads that are
  // waited for
  auto sync = [&](int lax) NIMBLE_INLINE {
    constexpr int MOST = FLIGHT + STORES < 63 ? FLIGHT + STORES : 63;
    asm volatile(
        "s_waitcnt lgkmcnt(0)\n\t"
        "s_cmp_eq_u32 %0, 0\n\t"
        "s_cbranch_scc0 .Lnimble_product_lax_%=\n\t"
        "s_waitcnt vmcnt(%2)\n"
        ".Lnimble_product_lax_%=:\n\t"
        "s_waitcnt vmcnt(%1)\n" ::"s"(__builtin_amdgcn_readfirstlane(lax)),
        "n"(MOST), "n"(FLIGHT)
        : "memory", "scc");
    __syncthreads();
  };
  // One stage.  FIRST: of a tile, its products start from zero.
  auto stage = [&](auto first_tag, int slot, int next, int last, int lax1, int lax2) NIMBLE_INLINE {
    constexpr bool FIRST = decltype(first_tag)::value;
    const uint32_t dst = lds0 + slot * SLOT;
    // TH x G tiles over the stage's 128 bytes, from the stage's product number n0 on; in between `nrd` fragment reads, then the
    // loads u0 ... u0 + nld - 1
    auto quarter = [&](auto& x, auto& w, auto th_tag, auto j0_tag, auto i0_tag, auto n0_tag, auto rd, auto nrd_tag, auto u0_tag,
                       auto nld_tag) NIMBLE_INLINE {
      constexpr int TH = decltype(th_tag)::value, N = 2 * G * TH, j0 = decltype(j0_tag)::value, i0 = decltype(i0_tag)::value;
      constexpr int n0 = decltype(n0_tag)::value, nrd = decltype(nrd_tag)::value, u0 = decltype(u0_tag)::value;
      constexpr int nops = nrd + decltype(nld_tag)::value;
      each<0, N>([&](auto n_tag) NIMBLE_INLINE {
        constexpr int n = decltype(n_tag)::value, kh = n / (G * TH), i = n / TH % G, j = i & 1 ? TH - 1 - n % TH : n % TH;
        constexpr bool zero = FIRST && kh == 0;
        Acc& sum = acc[i0 + i][j0 + j];
        constexpr int m0 = (n * nops + N - 1) / N, m1 = ((n + 1) * nops + N - 1) / N;
        constexpr int load0 = m0 > nrd ? m0 : nrd;  // loads of this gap: the last one goes behind the MFMA
        each<m0, (m1 < nrd ? m1 : nrd)>([&](auto m) NIMBLE_INLINE {
          rd(m);
          asm volatile("" ::: "memory");
        });
        constexpr int u = m1 > load0 && n0 + n != MFMAS - 1 ? u0 + m1 - 1 - nrd : -1;
        each<load0, (u >= 0 ? m1 - 1 : m1)>([&](auto m) NIMBLE_INLINE {
          constexpr int l = u0 + decltype(m)::value - nrd;
          dma16_buffer(off[l], src(l), at, dst + lds_off[l]);
        });
        if constexpr (n0 + n == MFMAS - 1)
          mfma_in_place_last(sum, w[i][kh], x[j][kh], last);
        else if constexpr (u >= 0)
          mfma_in_place_load<zero>(sum, w[i][kh], x[j][kh], off[u], src(u), at, dst, lds_off[u]);
        else
          mfma_in_place<zero>(sum, w[i][kh], x[j][kh]);
      });
    };
    sync(lax1);
    quarter(xa0, wb0, Int<H0>{}, Int<0>{}, Int<0>{}, Int<0>{}, [&](int m) NIMBLE_INLINE { rd_b1(slot, m); }, Int<TN>{}, Int<0>{}, Int<H0>{});
    quarter(xa0, wb1, Int<H0>{}, Int<0>{}, Int<G>{}, Int<2 * G * H0>{}, [&](int m) NIMBLE_INLINE { rd_a1(slot, m); }, Int<2 * H1>{}, Int<H0>{},
            Int<G>{});
    sync(lax2);
    quarter(xa1, wb0, Int<H1>{}, Int<H0>{}, Int<0>{}, Int<4 * G * H0>{}, [&](int m) NIMBLE_INLINE { rd_a0(next, m); }, Int<2 * H0>{},
            Int<H0 + G>{}, Int<G>{});
    quarter(xa1, wb1, Int<H1>{}, Int<H0>{}, Int<G>{}, Int<4 * G * H0 + 2 * G * H1>{}, [&](int m) NIMBLE_INLINE { rd_b0(next, m); }, Int<TN>{},
            Int<H0 + TN>{}, Int<H1>{});
  };
  at = S * 128;
  int slot = 0, parity = 0;
  bool stored = false;  // the tile before has issued its stores behind this one's first S stages
  const bool tail = !tight && (g.row_bytes & 127) != 0;
  for (int t = blockIdx.x;; t += gridDim.x) {
    const bool follows = t + (int)gridDim.x < tiles_total;
    // Stage ks loads stage ks + S of this tile: of its last one the pieces past the end of K are zeros; behind it come the next
    // tile's first ones (there is none: nothing is read).
    auto run_stage = [&](int ks, auto first_tag) NIMBLE_INLINE {
      if (tail && ks == KS - S - 1) set_off(KS - 1);
      if (tight) set_off(ks);  // (it loads that stage of the next tile)
      if (ks == KS - S) {
        at = 0;
        if (tail) set_off(0);
        a_src = b_src = descriptor(g.x, 0);
        if (follows) {
          tile_at(t + (int)gridDim.x, next_tile);
          a_src = a_desc(next_tile);
          b_src = b_desc(next_tile);
        }
      }
      const int next = slot + 1 == S ? 0 : slot + 1;
      stage(first_tag, slot, next, ks + 1 >= KS, stored && ks < S, stored && ks < S - 1);
      slot = next;
      at += 128;
    };
    run_stage(0, std::true_type{});
    for (int ks = 1; ks < KS; ++ks) run_stage(ks, std::false_type{});
    // (not before this tile's barriers: the values come where those of the tile before were)
    if (follows) fetch_values(next_tile, values + (parity ^ 1));
    if (g.epilogue == NIMBLE_EPI_BIAS_GELU_ERF)
      finish(tile, values[parity], std::true_type{});
    else
      finish(tile, values[parity], std::false_type{});
    if (!follows) break;
    stored = true;
    tile = next_tile;
    parity ^= 1;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

}  // namespace nimble
#endif
