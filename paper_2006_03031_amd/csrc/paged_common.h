// Attention of new rows over a paged cache: what each workgroup does, the parts of long sequences, and what the kernels share.
#ifndef NIMBLE_PAGED_COMMON_H_
#define NIMBLE_PAGED_COMMON_H_
#include <type_traits>

#include "cache_device.h"

namespace nimble {

struct PagedArgs {
  CacheArgs cache;
  SequencesArgs seqs;
  const uint16_t* q;
  uint16_t* o;
  long long q_stride;
  int heads, group;    // query heads, and those that share a key head
  int window;          // 0: none
  float a2;            // alpha log2 e
  float* part;         // [slots][rows][D] sums of parts, not divided
  float2* stat;        // [slots][rows] their largest score (base 2) and sum of probabilities
  int* items;          // [0]: tiles that were cut, then 8 words each
  int slots, target_units, join_rows;  // join_rows: the most rows of a tile
};

constexpr float kNothing = -3.0e38f;  // the reference of a row that has seen no key yet

// ---------------------------------------------------------------------------
// What a workgroup does: a tile of ROWS rows of one sequence and one head of the cache, or a part of the keys that it sees.
// The rows of a (sequence, head) are its tokens times the query heads that share the head, row = token * group + query head: all of them
// meet the same keys.  Only the device knows the lengths, so it is the device that cuts: the key blocks of all tiles together, divided by
// the units that fill the chip, are the most that one part takes, and a tile that has more is cut into equal parts.  Every wave works
// this out for itself from all lengths, 64 sequences a step.  Heavy tiles of a sequence come first, the heads of the cache innermost: their
// workgroups go to the XCDs in turn, so that the tiles which read one head's keys share an L2.
// ---------------------------------------------------------------------------
struct PagedUnit {
  Sequence seq;
  int s, head, tile, tiles;
  int part, parts;
  int slot, item;  // in the workspace, where parts > 1
};

template <int ROWS, int KEYS>
__device__ __forceinline__ void tile_work(const PagedArgs& g, const Sequence& q, int& tiles, int& blocks) {
  tiles = (q.n * g.group + ROWS - 1) / ROWS;  // (at most 2^24 rows of 2^6 heads and so on: checked by the host)
  int keys = q.length;
  if (g.window > 0 && g.window + ROWS < keys) keys = g.window + ROWS;
  blocks = tiles ? (keys + KEYS - 1) / KEYS : 0;
}

// The most blocks of one part.  The same in every lane of every wave of a call.
template <int ROWS, int KEYS, int LEAST>
__device__ __forceinline__ int part_blocks(const PagedArgs& g) {
  const int lane = threadIdx.x & 63;
  float total = 0;
  for (int base = 0; base < g.seqs.count; base += 64) {
    const int s = base + lane;
    if (s < g.seqs.count) {
      int tiles, blocks;
      tile_work<ROWS, KEYS>(g, sequence_of(g.seqs, s, g.cache.page_shift), tiles, blocks);
      total += (float)tiles * (float)blocks;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
  const float most = ceilf(total * (float)g.cache.kv_heads / (float)g.target_units) + 1.0f;
  return most < (float)LEAST ? LEAST : most > 1.0e9f ? 1000000000 : (int)most;
}

template <int ROWS, int KEYS, int LEAST>
__device__ __forceinline__ bool find_unit(const PagedArgs& g, unsigned unit, PagedUnit& u, int& items) {
  const int lane = threadIdx.x & 63, G = g.cache.kv_heads;
  const int most = g.slots ? part_blocks<ROWS, KEYS, LEAST>(g) : 1000000000;
  const unsigned want = unit / G;
  u.head = (int)(unit - want * G);
  unsigned units = 0, cut_units = 0, cut_tiles = 0;  // of the sequences ahead
  bool found = false;
  for (int base = 0; base < g.seqs.count && (!found || unit == 0); base += 64) {
    const int s = base + lane;
    Sequence q{0, 0, 0};
    int tiles = 0, blocks = 0;
    if (s < g.seqs.count) {
      q = sequence_of(g.seqs, s, g.cache.page_shift);
      tile_work<ROWS, KEYS>(g, q, tiles, blocks);
    }
    const int parts = blocks > most ? (blocks + most - 1) / most : 1;
    const unsigned mine = (unsigned)tiles * parts, mine_cut = parts > 1 ? mine : 0, tiles_cut = parts > 1 ? tiles : 0;
    unsigned a = mine, b = mine_cut, c = tiles_cut;  // inclusive sums
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const unsigned ua = __shfl_up(a, o, 64), ub = __shfl_up(b, o, 64), uc = __shfl_up(c, o, 64);
      if (lane >= o) a += ua, b += ub, c += uc;
    }
    const unsigned long long here = __ballot(units + a > want);
    if (!found && here) {
      const int l = __ffsll((unsigned long long)here) - 1;
      auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
      const unsigned before = units + (unsigned)of((int)(a - mine));
      u.s = base + l;
      u.seq.first = of(q.first);
      u.seq.n = of(q.n);
      u.seq.length = of(q.length);
      u.tiles = of(tiles);
      u.parts = of(parts);
      const int rest = (int)(want - before);
      const int back = rest / u.parts;
      u.tile = u.tiles - 1 - back;
      u.part = rest - back * u.parts;
      u.slot = (int)((cut_units + (unsigned)of((int)(b - mine_cut)) + rest) * G + u.head);
      u.item = (int)((cut_tiles + (unsigned)of((int)(c - tiles_cut)) + back) * G + u.head);
      found = true;
    }
    units += (unsigned)__builtin_amdgcn_readlane((int)a, 63);
    cut_units += (unsigned)__builtin_amdgcn_readlane((int)b, 63);
    cut_tiles += (unsigned)__builtin_amdgcn_readlane((int)c, 63);
  }
  items = (int)cut_tiles * G;  // (of all sequences where unit = 0, which looks at all)
  return found;
}

// The keys of a tile, and of one part of it, in blocks.
template <int ROWS, int KEYS>
__device__ __forceinline__ void unit_keys(const PagedArgs& g, const PagedUnit& u, int& low, int& high, int& block0, int& block1) {
  const int m0 = u.tile * ROWS, rows = u.seq.n * g.group, m1 = (m0 + ROWS < rows ? m0 + ROWS : rows) - 1;
  const int before = u.seq.length - u.seq.n;
  high = before + m1 / g.group;                                             // the last key that a row of the tile sees
  low = 0;
  if (g.window > 0) {
    low = before + m0 / g.group - g.window + 1;                             // and the first
    if (low < 0) low = 0;
  }
  low = __builtin_amdgcn_readfirstlane(low);
  high = __builtin_amdgcn_readfirstlane(high);
  if (high < 0) {
    block0 = block1 = 0;
    return;
  }
  const int b0 = low / KEYS, nb = high / KEYS + 1 - b0, q = nb / u.parts, r = nb - q * u.parts;  // (the first r parts have one more)
  block0 = __builtin_amdgcn_readfirstlane(b0 + u.part * q + (u.part < r ? u.part : r));
  block1 = __builtin_amdgcn_readfirstlane(block0 + q + (u.part < r ? 1 : 0));
}

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
  const int token = m / g.group;
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
  if (u.parts > 1) {
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

// What the second launch has to know of a tile that was cut.
__device__ __forceinline__ void put_item(const PagedArgs& g, const PagedUnit& u) {
  int* item = g.items + (1 + u.item) * kPagedItemWords;
  item[0] = u.slot, item[1] = u.parts, item[2] = u.tile, item[3] = u.head;
  item[4] = u.seq.first, item[5] = u.seq.n, item[6] = u.seq.length, item[7] = g.cache.kv_heads;  // (slots of a tile's parts are kv_heads apart)
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
// The parts of a row joined, in the order of the parts: o = sum_x 2^(ref_x - top) part_x / sum_x 2^(ref_x - top) sum_x.  A wave a row; where there
// are fewer rows than workgroups a workgroup a row, whose waves take every fourth part.  A lane looks at one part's (ref, sum) and the wave at its
// sums one part after the other, 8 loads at a time.
// ---------------------------------------------------------------------------
template <int ROWS, int D>
__global__ void __launch_bounds__(256) paged_join_kernel(PagedArgs g) {
  constexpr int P = D / 64;
  typedef float Piece __attribute__((ext_vector_type(P)));
  __shared__ float2 wave_stat[4];
  __shared__ Piece wave_sums[4][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long count = (long long)g.items[0] * g.join_rows;
  const bool together = count <= gridDim.x;
  const int step = together ? 4 : 1;
  for (long long at = together ? blockIdx.x : (long long)blockIdx.x * 4 + wave; at < count; at += together ? gridDim.x : 4ll * gridDim.x) {
    const int* item = g.items + (1 + at / g.join_rows) * kPagedItemWords;
    const int row = (int)(at % g.join_rows);
    const int slot = item[0], parts = item[1], apart = item[7], mm = item[2] * ROWS + row;
    if (mm >= item[5] * g.group) continue;  // (the same in the whole workgroup where its waves work together)
    float top = kNothing, total = 0.f;
    Piece acc{};
    for (int x0 = together ? wave : 0; x0 < parts; x0 += 64 * step) {
      const int x = x0 + lane * step;
      const float2 st = x < parts ? g.stat[(long long)(slot + x * apart) * ROWS + row] : make_float2(kNothing, 0.f);
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
      const int n = (parts - x0 + step - 1) / step < 64 ? (parts - x0 + step - 1) / step : 64;
      for (int y0 = 0; y0 < n; y0 += 8) {
        Piece v[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const int part = x0 + (y0 + y < n ? y0 + y : n - 1) * step;
          v[y] = *(const Piece*)(g.part + ((long long)(slot + part * apart) * ROWS + row) * D + lane * P);
        }
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
    const int tok = mm / g.group;
    const float inv = item[6] - item[5] + tok < 0 ? 0.f : 1.0f / total;
    u16* o = g.o + ((long long)(item[4] + tok) * g.heads + item[3] * g.group + mm - tok * g.group) * D + lane * P;
    if constexpr (P == 2)
      *(uint32_t*)o = pack_bf16x2(acc[0] * inv, acc[1] * inv);
    else
      *o = f2bf(acc[0] * inv);
  }
}

}  // namespace nimble
#endif
