// Attention of new rows over a paged cache: what the kernels share, and the join of the parts of long sequences.
#ifndef NIMBLE_PAGED_COMMON_H_
#define NIMBLE_PAGED_COMMON_H_
#include "paged_work.h"

namespace nimble {

// A pointer that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const unsigned char* uniform_pointer(const unsigned char* p) {
  const uint64_t a = (uint64_t)p;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
  return (const unsigned char*)(((uint64_t)hi << 32) | lo);
}

// One row of a unit, key by key, 64 at a time: for the units in whose results an infinity or a NaN turned up.  The matrix products multiply
// what a row does not see by 0, which an infinite or NaN value there turns into NaN; here it is not looked at.
// A lane holds elements lane and lane + 64 of the sum; ref is in base 2.  Writes the row's part, or the row.
template <int ROWS, int D>
__device__ __forceinline__ void careful_row(const PagedArgs& g, const PagedUnit& u, int m, int key0, int key1) {
  constexpr int P = D / 64;
  const int lane = threadIdx.x & 63;
  const int token = divided(m, g.by_group);
  const int p = u.seq.length - u.seq.n + token;
  int first = g.window > 0 ? p - g.window + 1 : 0, last = p;
  if (first < key0) first = key0;
  if (last >= key1) last = key1 - 1;
  const u16* q = g.q + (long long)(u.seq.first + token) * g.q_stride + (u.head * g.group + m - token * g.group) * D;
  float ref = kNothing, sum = 0, acc[P];
#pragma unroll
  for (int i = 0; i < P; ++i) acc[i] = 0;
  auto row_of = [&](int key) {
    unsigned page = (unsigned)g.seqs.pages[(long long)u.s * g.seqs.width + (key >> g.cache.page_shift)];
    page = page < g.cache.pages ? page : g.cache.pages - 1;
    return (((long long)page * g.cache.kv_heads + u.head) << g.cache.page_shift) + (key & ((1 << g.cache.page_shift) - 1));
  };
  for (int j = first; j <= last; j += 64) {
    const bool mine = j + lane <= last;
    long long row = 0;
    float s = -INFINITY;
    if (mine) {
      row = row_of(j + lane);
      const u16* k = (const u16*)g.cache.k + row * D;
      s = 0;
      for (int d = 0; d < D; ++d) s = fmaf(bf2f(q[d]), bf2f(k[d]), s);
      s *= g.a2;
    }
    float top = fmaxf(ref, s);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float e = mine ? __builtin_amdgcn_exp2f(s - top) : 0.0f, back = __builtin_amdgcn_exp2f(ref - top);
    float t = e;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o, 64);
    sum = sum * back + t;
#pragma unroll
    for (int i = 0; i < P; ++i) acc[i] *= back;
    ref = top;
    const int n = last - j + 1 < 64 ? last - j + 1 : 64;
    for (int x = 0; x < n; ++x) {
      const float px = __shfl(e, x, 64);
      const long long rx = __shfl(row, x, 64);
#pragma unroll
      for (int i = 0; i < P; ++i) acc[i] = fmaf(px, bf2f(((const u16*)g.cache.v)[rx * D + i * 64 + lane]), acc[i]);
    }
  }
  if (u.slot >= 0) {
    const long long to = (long long)u.slot * ROWS + m - u.tile * ROWS;
#pragma unroll
    for (int i = 0; i < P; ++i) g.part[to * D + i * 64 + lane] = acc[i];
    if (lane == 0) g.stat[to] = make_float2(ref, sum);
    return;
  }
  const float inv = p < 0 ? 0.f : 1.0f / sum;
  u16* o = g.o + ((long long)(u.seq.first + token) * g.heads + u.head * g.group + m - token * g.group) * D;
#pragma unroll
  for (int i = 0; i < P; ++i) o[i * 64 + lane] = f2bf(acc[i] * inv);
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

typedef int i32x2 __attribute__((ext_vector_type(2)));
// Transposing LDS read of bytes: the 16 lanes of a group each name 8 bytes, taken as 8 rows of 16 (lanes 2 r, 2 r + 1 hold row r); lane i
// of the group receives column i.
__device__ __forceinline__ uint2 lds_read_tr8(uint32_t lds_addr) {
  typedef __attribute__((address_space(3))) i32x2* ptr;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((ptr)(uintptr_t)lds_addr));
}
__device__ __forceinline__ void dma4(const void* g, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off\n" ::"v"(g), "s"(lds_addr) : "memory", "m0");
}
// Four codes as bf16.
__device__ __forceinline__ uint2 codes_to_bf16(uint32_t w) {
  const float a = (float)(signed char)w, b = (float)(signed char)(w >> 8), c = (float)(signed char)(w >> 16), d = (float)((int)w >> 24);
  return make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}

// ---------------------------------------------------------------------------
// The parts of a row joined, in the order of the parts: o = sum_x 2^(ref_x - top) part_x / sum_x 2^(ref_x - top) sum_x.  A wave a row; with more
// than 8 parts, and rows few enough that each has a workgroup, a workgroup a row, whose waves take every fourth
// part.  A lane looks at one part's (ref, sum) and the wave at its sums one part after the other, 8 loads at a time.  Bound by latency: 4.6 to 5.1 us, of
// 32 rows of 256 parts as of 128 rows of 2.
// ---------------------------------------------------------------------------
template <int ROWS, int D>
__global__ void __launch_bounds__(256) paged_join_kernel(PagedArgs g) {
  constexpr int P = D / 64, MANY = 8;
  typedef float Piece __attribute__((ext_vector_type(P)));
  __shared__ float2 wave_stat[4];
  __shared__ Piece wave_sums[4][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (the grid is as long as the table of tiles can be; an entry is read with the number of entries, not behind it)
  const int* entry = g.items + (1 + blockIdx.x) * kPagedItemWords;
  int item[9], count = g.items[0];
#pragma unroll
  for (int x = 0; x < 9; ++x) item[x] = entry[x];
  const int parts = item[0], slot = item[1], second = item[2], apart = item[3], tile = item[4], head = item[5];
  if ((int)blockIdx.x >= count || parts < 2) return;
  const int left = item[7] * g.group - tile * ROWS, rows = left < ROWS ? left : ROWS;
  const bool together = parts > MANY && rows <= (int)gridDim.y;
  const int step = together ? 4 : 1;
  for (int row = blockIdx.y + (together ? 0 : wave * gridDim.y); row < rows; row += together ? gridDim.y : 4 * gridDim.y) {
    float top = kNothing, total = 0.f;
    Piece acc{};
    auto place = [&](int x) { return (long long)(x ? second + (x - 1) * apart : slot) * ROWS + row; };
    for (int x0 = together ? wave : 0; x0 < parts; x0 += 64 * step) {
      const int x = x0 + lane * step;
      const float2 st = x < parts ? g.stat[place(x)] : make_float2(kNothing, 0.f);
      const int n = (parts - x0 + step - 1) / step < 64 ? (parts - x0 + step - 1) / step : 64;
      Piece v[8];
      auto load = [&](int y0) {
#pragma unroll
        for (int y = 0; y < 8; ++y) v[y] = *(const Piece*)(g.part + place(x0 + (y0 + y < n ? y0 + y : n - 1) * step) * D + lane * P);
      };
      load(0);
      float next = fmaxf(top, st.x);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) next = fmaxf(next, __shfl_xor(next, o, 64));
      const float back = __builtin_amdgcn_exp2f(top - next), scale = __builtin_amdgcn_exp2f(st.x - next);
      float sum = st.y * scale;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      total = total * back + sum;
      acc *= back;
      top = next;
      for (int y0 = 0; y0 < n; y0 += 8) {
        if (y0) load(y0);
#pragma unroll
        for (int y = 0; y < 8; ++y)
          if (y0 + y < n) acc += v[y] * __shfl(scale, y0 + y, 64);
      }
    }
    if (together) {
      __syncthreads();
      if (lane == 0) wave_stat[wave] = make_float2(top, total);
      wave_sums[wave][lane] = acc;
      __syncthreads();
      if (wave > 0) continue;
      float t = kNothing;
#pragma unroll
      for (int w = 0; w < 4; ++w) t = fmaxf(t, wave_stat[w].x);
      total = 0.f;
      acc = Piece{};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float scale = __builtin_amdgcn_exp2f(wave_stat[w].x - t);
        total += wave_stat[w].y * scale;
        acc += wave_sums[w][lane] * scale;
      }
    }
    const int mm = tile * ROWS + row, tok = divided(mm, g.by_group);
    const float inv = item[8] - item[7] + tok < 0 ? 0.f : 1.0f / total;
    u16* o = g.o + ((long long)(item[6] + tok) * g.heads + head * g.group + mm - tok * g.group) * D + lane * P;
    if constexpr (P == 2)
      *(uint32_t*)o = pack_bf16x2(acc[0] * inv, acc[1] * inv);
    else
      *o = f2bf(acc[0] * inv);
  }
}

}  // namespace nimble
#endif
