// Products whose rows fall into groups with a weight each, at offsets that only the device knows: the map from workgroups to
// tiles, the epilogue, and the kernel for operands of any alignment.
#ifndef NIMBLE_GROUPED_KERNEL_H_
#define NIMBLE_GROUPED_KERNEL_H_
#include <type_traits>

#include "device_common.h"
#include "grouped_internal.h"

namespace nimble {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// The matrix instruction of an element type.  Either takes 16 bytes of one row per lane (row lane & 15, piece lane >> 4), 64 bytes
// of K per instruction, and leaves four consecutive n of one m in a lane: the kernels differ in nothing else.
struct OfBf16 {
  typedef f32x4 Acc;
  static constexpr bool kInt8 = false;
  static __device__ __forceinline__ Acc mfma(uint4 w, uint4 x, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), as_bf16x8(x), c, 0, 0, 0);
  }
};
struct OfInt8 {
  typedef i32x4 Acc;
  static constexpr bool kInt8 = true;
  static __device__ __forceinline__ Acc mfma(uint4 w, uint4 x, Acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, x), c, 0, 0, 0);
  }
};

typedef int rsrc_t __attribute__((ext_vector_type(4)));
// The first `bytes` (below 2^31) from p on.
__device__ __forceinline__ rsrc_t descriptor(const void* p, uint32_t bytes) {
  const uint64_t a = (uint64_t)p;
  return rsrc_t{__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32)),
                __builtin_amdgcn_readfirstlane((int)bytes), 0x00027000};
}
// 16 bytes per lane from the descriptor's byte voff + soff to LDS; past its end zeros.
__device__ __forceinline__ void dma16_buffer(uint32_t voff, rsrc_t rsrc, uint32_t soff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(voff), "s"(rsrc), "s"(soff),
               "s"(lds_addr)
               : "memory", "m0");
}
__device__ __forceinline__ void dma4_buffer(uint32_t voff, rsrc_t rsrc, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "s"(lds_addr)
               : "memory", "m0");
}

// Where the tiles of a launch are.  With groups, tile rows are counted group after group, a group of m rows has ceil(m / BM) of
// them; `ends[e]` is their number up to and with group e, `starts[e]` the group's first row.  Offsets are brought into [0, rows], and one
// that falls to the largest before it: whatever they hold, groups do not overlap, no access leaves the operands, and
// there are no more tiles than the host allowed for.
// (MOST = 0: no groups.)
template <int MOST>
struct GroupMap {
  int ends[MOST + 1];
  int starts[MOST + 1];
};
static_assert(sizeof(GroupMap<kMostGroups>) == group_map_bytes(kMostGroups), "LDS of the map as the host takes it");
// Filled by the first wave; the caller's barrier publishes it.
template <int BM, int MOST>
__device__ __forceinline__ void map_groups(const ProductArgs& g, GroupMap<MOST>& map) {
  if (threadIdx.x >= 64) return;
  const int lane = (int)threadIdx.x;
  int tiles = 0, furthest = 0;
  for (int base = 0; base < g.groups; base += 64) {
    const int e = base + lane;
    int first = 0, end = 0;
    if (e < g.groups) {
      first = (int)min(max(g.offsets[e], 0ll), g.rows);
      end = (int)min(max(g.offsets[e + 1], 0ll), g.rows);
    }
    first = max(first, furthest);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(first, o, 64);
      if (lane >= o) first = max(first, up);
    }
    end = e < g.groups ? max(end, first) : first;
    furthest = max(furthest, __shfl(end, 63, 64));
    int n = (int)(((long long)end - first + BM - 1) / BM);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(n, o, 64);
      if (lane >= o) n += up;
    }
    n += tiles;
    if (e < g.groups) {
      map.ends[e] = n;
      map.starts[e] = first;
      if (e == g.groups - 1) map.starts[g.groups] = end;
    }
    tiles = __shfl(n, 63, 64);
  }
}
// The group of tile row t (t < ends[groups - 1]): as many groups end at or before it.  The same in all lanes.
template <int MOST>
__device__ __forceinline__ int group_of_tile_row(const GroupMap<MOST>& map, int groups, int t) {
  int e = 0;
  for (int base = 0; base < groups; base += 64) {
    const int i = base + (int)(threadIdx.x & 63);
    e += __popcll(__ballot(i < groups && map.ends[i] <= t));
  }
  return e;
}

struct ProductTile {
  int row0;  // first row of the tile
  int rows;  // how many, at most BM
  int group, n0;
};

// The 16 bytes at byte `at` of a row; past the end of the row zero.  Any alignment.
__device__ __forceinline__ uint4 load16(const unsigned char* row, int at, int row_bytes) {
  uint4 v = make_uint4(0, 0, 0, 0);
  const int left = row_bytes - at;
  if (left >= 16) {
    __builtin_memcpy(&v, row + at, 16);
  } else if (left > 0 && row_bytes >= 16) {  // the row's last 16 bytes, moved down
    __builtin_memcpy(&v, row + row_bytes - 16, 16);
    const uint64_t lo = ((uint64_t)v.y << 32) | v.x, hi = ((uint64_t)v.w << 32) | v.z;
    const int sh = 8 * (16 - left);  // 8 .. 120 bits
    const uint64_t rlo = sh < 64 ? (lo >> sh) | (hi << (64 - sh)) : hi >> (sh - 64);
    const uint64_t rhi = sh < 64 ? hi >> sh : 0;
    v = make_uint4((uint32_t)rlo, (uint32_t)(rlo >> 32), (uint32_t)rhi, (uint32_t)(rhi >> 32));
  } else if (left > 0) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int b = 0; b < 15; ++b)
      if (b < left) w[b >> 2] |= (uint32_t)row[at + b] << (8 * (b & 3));
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}

// 16 bytes from an address that is a whole number of words.
__device__ __forceinline__ uint4 load16_at_word(const void* p) {
  uint4 v;
  __builtin_memcpy(&v, __builtin_assume_aligned(p, 4), 16);
  return v;
}
// 16 bytes from any address, by words that start at whole words: loads that do not come from the L2 at a third of the rate.  Up to three
// bytes ahead of them (of the row before) and three behind them are read too.
__device__ __forceinline__ uint4 load16_words(const unsigned char* p) {
  const uint32_t by = (uint32_t)(uintptr_t)p & 3u;
  const uint32_t* a = (const uint32_t*)(p - by);
  const uint4 v = load16_at_word(a);
  const uint32_t next = a[by ? 4 : 3];
  return make_uint4(__builtin_amdgcn_alignbyte(v.y, v.x, by), __builtin_amdgcn_alignbyte(v.z, v.y, by),
                    __builtin_amdgcn_alignbyte(v.w, v.z, by), __builtin_amdgcn_alignbyte(next, v.w, by));
}

// gelu(v) = v/2 (1 + erf(v / sqrt 2)) = max(v, 0) - |v| Q(|v|), Q the upper tail of the normal distribution.  log2 Q is smooth for
// x >= 0 and -1 at 0, so Q is 2^P(x) with a polynomial P: one transcendental instruction per value, and the roundings of a small tail do not
// reach a result that is not small.  P is a minimax fit to log2 Q on [0, 8].  With the roundings of f32 and of the hardware's exp2 (1 ulp) a
// result is off by at most
//   f32 outputs,  degree 10, the fit's error weighted by 1 / (1 + (x/2)^6):   2^-21 of itself for v >= 0, 2^-21 (1 + (v/2)^6) for -8 <= v < 0;
//   bf16 outputs, degree 8, weighted by 1 / (1 + (x/1.4)^6):                  2^-20 of itself for v >= 0, 2^-20 (1 + (v/1.4)^6) for -8 <= v < 0,
// 1/2000 of half a step of bf16 where results are not small: of 100000 results from values of spread 0.65 four are not the rounded exact ones, one
// of them with degree 10.  (Two steps of the polynomial are 1.9 us of the 47.4 of 8177 x 4096 x 1024 in 8 bits, 4 of 114 of 16354 rows over 8 groups.)
// Below -8 P falls on to minus infinity and the result stays under 2^-46; above 8, where it is v, x stays 8, so that infinity less nothing is infinity.
// NaN stays NaN, and minus infinity gives NaN as the formula does.
//   N values side by side, step by step (the empty statements keep the N results of a step together), as epilogue_of does it.
template <bool F32, int N>
__device__ __forceinline__ void gelu_of(float (&v)[N]) {
  constexpr int kDegree = F32 ? 10 : 8;
  constexpr float kTail32[11] = {-1.0f,           -1.15110886f,    -0.459177405f,  -0.0525782481f,  0.00715400605f, -0.000172875938f,
                                 -0.000194635781f, 5.13012637e-05f, -6.58381487e-06f, 4.4570379e-07f, -1.26317756e-08f};
  constexpr float kTail16[9] = {-1.0f, -1.15111983f, -0.459074169f, -0.0529038422f, 0.00763690891f,
                                -0.000555595732f, -2.37187851e-05f, 7.77410787e-06f, -4.18191178e-07f};
  float x[N], p[N];
  auto together = [&](float (&y)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(y[i]));
  };
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = fabsf(__builtin_elementwise_minimum(v[i], 8.0f)), p[i] = F32 ? kTail32[10] : kTail16[8];
#pragma unroll
  for (int k = kDegree - 1; k >= 0; --k) {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = fmaf(p[i], x[i], F32 ? kTail32[k] : kTail16[k < 8 ? k : 8]);
    together(p);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = __builtin_amdgcn_exp2f(p[i]);
  together(p);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = fmaf(-x[i], p[i], __builtin_elementwise_maximum(v[i], 0.0f));
}

// Four consecutive outputs of a row from n on, as many as there are; `v` is scaled and has its bias.
__device__ __forceinline__ void store4(const ProductArgs& g, float (&v)[4], long long row, int n) {
  const int n4 = g.N - n;
  const bool gelu = g.epilogue == NIMBLE_EPI_BIAS_GELU_ERF;
  const long long at = row * g.N + n;
  if (g.out_f32) {
    if (gelu) gelu_of<true>(v);
    float* y = (float*)g.y + at;
    if (n4 >= 4) {
      __builtin_memcpy(y, v, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < n4) y[e] = v[e];
    }
  } else {
    if (gelu) gelu_of<false>(v);
    u16* y = (u16*)g.y + at;
    if (n4 >= 4) {
      const uint2 pk = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
      __builtin_memcpy(y, &pk, 8);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < n4) y[e] = f2bf(v[e]);
    }
  }
}

// The tile at tile row t and tile column tn; false where there is none (fewer tile rows than the host had to allow for).
template <int BM, int BN, int MOST>
__device__ __forceinline__ bool find_tile(const ProductArgs& g, const GroupMap<MOST>& map, int t, int tn, ProductTile& tile) {
  int first = t * BM, end = (int)g.rows;
  tile.n0 = tn * BN;
  tile.group = 0;
  if (MOST > 0) {
    if (t >= map.ends[g.groups - 1]) return false;
    tile.group = group_of_tile_row(map, g.groups, t);
    first = map.starts[tile.group] + (t - (tile.group ? map.ends[tile.group - 1] : 0)) * BM;
    end = map.starts[tile.group + 1];
  }
  tile.row0 = __builtin_amdgcn_readfirstlane(first);
  tile.rows = __builtin_amdgcn_readfirstlane(min(end - first, BM));
  return true;
}

// ---------------------------------------------------------------------------
// Any alignment: TM x TN blocks of 16 x 16 per workgroup, KW waves that take pieces of 64 bytes of K in turn, operands from
// memory straight into the registers that the matrix instruction reads; the waves' sums meet in LDS.  Bound: the L2s' answers to loads of rows
// that start anywhere.  Loaded by whole words and shifted into place, not at their own addresses: 8177 x 4096 x 1003 in 8 bits 218 us,
// 282; 200 x 1024 x 4099 27.5, 48.4; 4000 rows over 8 groups x 1024 x 1001 in bf16 61, 87.  A second register set for the pieces ahead took a
// workgroup's place on the compute unit: 365 us.
// ---------------------------------------------------------------------------
template <typename T, int GROUPS, int TM, int TN, int KW>
__global__ void __launch_bounds__(KW * 64) product_direct_kernel(ProductArgs g, unsigned tiles, unsigned tiles_n) {
  constexpr int BM = 16 * TM, BN = 16 * TN;
  typedef typename T::Acc Acc;
  __shared__ GroupMap<GROUPS> map;
  __shared__ __attribute__((aligned(16))) Acc sums[KW][TM * TN * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr_row = lane & 15, fr_at = (lane >> 4) * 16;
  if (GROUPS) {
    map_groups<BM>(g, map);
    __syncthreads();
  }
  for (unsigned b = blockIdx.x; b < tiles; b += gridDim.x) {
    ProductTile tile;
    const unsigned t = b / tiles_n;
    if (!find_tile<BM, BN>(g, map, (int)t, (int)(b - t * tiles_n), tile)) return;
    const unsigned char *xp[TM], *wp[TN];
#pragma unroll
    for (int j = 0; j < TM; ++j) xp[j] = g.x + ((long long)tile.row0 + min(16 * j + fr_row, tile.rows - 1)) * g.row_bytes;
#pragma unroll
    for (int i = 0; i < TN; ++i) wp[i] = g.w + ((long long)tile.group * g.N + min(tile.n0 + 16 * i + fr_row, g.N - 1)) * g.row_bytes;
    Acc acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = Acc{0, 0, 0, 0};
    uint4 x[TM], w[TN];
    int at = wave * 64;
    auto walk = [&](auto whole_words) {
      constexpr bool kWords = decltype(whole_words)::value;
      for (; at + 64 + (kWords ? 0 : 3) <= g.row_bytes; at += KW * 64) {
#pragma unroll
        for (int i = 0; i < TN; ++i) w[i] = kWords ? load16_at_word(wp[i] + at + fr_at) : load16_words(wp[i] + at + fr_at);
#pragma unroll
        for (int j = 0; j < TM; ++j) x[j] = kWords ? load16_at_word(xp[j] + at + fr_at) : load16_words(xp[j] + at + fr_at);
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j) acc[i][j] = T::mfma(w[i], x[j], acc[i][j]);
      }
    };
    if ((g.row_bytes & 3) == 0)
      walk(std::true_type{});
    else
      walk(std::false_type{});
    if (at < g.row_bytes) {
#pragma unroll
      for (int i = 0; i < TN; ++i) w[i] = load16(wp[i], at + fr_at, g.row_bytes);
#pragma unroll
      for (int j = 0; j < TM; ++j) x[j] = load16(xp[j], at + fr_at, g.row_bytes);
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = T::mfma(w[i], x[j], acc[i][j]);
    }
    if (b != blockIdx.x) __syncthreads();  // the tile before has been read
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) sums[wave][(i * TM + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < TM * TN * 64; o += KW * 64) {
      Acc s = sums[0][o];
#pragma unroll
      for (int k = 1; k < KW; ++k) s += sums[k][o];
      const int l = o & 63, block = o >> 6, i = block / TM, j = block % TM;
      const int r = 16 * j + (l & 15), n = tile.n0 + 16 * i + 4 * (l >> 4);
      if (r >= tile.rows || n >= g.N) continue;
      const long long row = (long long)tile.row0 + r;
      const float xs = T::kInt8 ? g.x_scale[row] : 1.0f;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const long long c = (long long)tile.group * g.N + min(n + e, g.N - 1);
        const float bias = g.epilogue != NIMBLE_EPI_NONE ? bf2f(g.bias[c]) : 0.0f;
        v[e] = T::kInt8 ? fmaf((float)s[e], xs * g.w_scale[c], bias) : (float)s[e] + bias;
      }
      store4(g, v, row, n);
    }
  }
}

}  // namespace nimble
#endif
