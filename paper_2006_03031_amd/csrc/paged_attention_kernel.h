// Attention of new rows over a paged cache.
#ifndef NIMBLE_PAGED_ATTENTION_KERNEL_H_
#define NIMBLE_PAGED_ATTENTION_KERNEL_H_
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
  int slots, target_units;
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
// A lane holds elements lane and lane + 64 of the sum; ref is in base 2.
template <int D>
__device__ __forceinline__ void careful_row(const PagedArgs& g, const PagedUnit& u, int m, int key0, int key1, float* out, float* row_stat) {
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
#pragma unroll
  for (int i = 0; i < P; ++i) out[i * 64 + lane] = acc[i];
  if (lane == 0) row_stat[0] = ref, row_stat[1] = sum;
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// ---------------------------------------------------------------------------
// Few rows: 16 of a (sequence, head) per workgroup, four waves that each take every fourth block of 32 keys and meet at the end.
//   scores:  MFMA 16x16x32, 16 keys on the A side, the 16 rows on the B side: lane (r, h) = (lane & 15, lane >> 4) holds, for row r, keys
//            16 t + 4 h + (0..3) of tile t = 0, 1.
//   P.V:     the 8 k slots of h are defined as the keys it holds, 4 of either tile, so that P stays in its lane; the values come out of
//            the row-major tile with the transposing LDS read (of 16 bits a piece, or of 8).
//   8 bits:  codes become bf16, which holds them exactly, behind the LDS reads; a key's scale multiplies its scores, a value's its
//            probability.  A lane reads 16 codes of a key row where it reads 8 elements of bf16, so that the elements of a
//            matrix instruction's k are taken from the row in another order, and those of q in the same.
//   Loads:   direct global->LDS loads into the wave's own ring of S blocks, waited for by count: no barrier in the loop.  16 keys lie in one
//            page, whose number is a scalar.  Chunk c of row r sits at c ^ swizzle(r).  Keys outside of what the tile sees repeat the
//            nearest one that it does.
// ---------------------------------------------------------------------------
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

template <int D, bool I8>
__global__ void __launch_bounds__(256) paged_tokens_kernel(PagedArgs g) {
  constexpr int ROWS = 16, KEYS = 32, LEAST = 8, WAVES = 4;
  constexpr int RB = D * (I8 ? 1 : 2);           // bytes of a key row
  constexpr int CH = RB / 16;                    // its chunks
  constexpr int PER = 1024 / RB;                 // rows of one load
  constexpr int LOADS = 16 / PER;                // loads of 16 rows
  constexpr int TILE = KEYS * RB;                // bytes of a block of K or V
  constexpr int SCALES = I8 ? 256 : 0;           // 32 scales of keys, 32 of values
  constexpr int SLOT = 2 * TILE + SCALES;
  constexpr int S = 2;
  constexpr int COUNT = 4 * LOADS + (I8 ? 1 : 0);  // loads of a block
  constexpr int RING = WAVES * S * SLOT, JOIN = WAVES * ROWS * D * 4;
  __shared__ __attribute__((aligned(256))) unsigned char lds[RING > JOIN ? RING : JOIN];
  __shared__ float2 stat[WAVES][ROWS];
  __shared__ int poisoned;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, h = lane >> 4;
  PagedUnit u;
  int items;
  const bool found = find_unit<ROWS, KEYS, LEAST>(g, blockIdx.x, u, items);
  if (g.slots && blockIdx.x == 0 && tid == 0) g.items[0] = found ? items : 0;
  if (!found) return;
  if (u.parts > 1 && (u.slot >= g.slots || u.item >= g.slots / 2)) return;  // (not with offsets that keep to their description)
  int low, high, block0, block1;
  unit_keys<ROWS, KEYS>(g, u, low, high, block0, block1);

  // this lane's row
  const int m = u.tile * ROWS + r16, rows = u.seq.n * g.group;
  const int m_ld = m < rows ? m : rows - 1;
  const int token = m_ld / g.group;
  const int pos = m < rows ? u.seq.length - u.seq.n + token : -1;
  const int first = g.window > 0 ? pos - g.window + 1 : 0;
  const u16* q = g.q + (long long)(u.seq.first + token) * g.q_stride + (u.head * g.group + m_ld - token * g.group) * D;
  bf16x8 qf[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const int at = I8 ? (i >> 1) * 64 + h * 16 + (i & 1) * 8 : i * 32 + h * 8;
    qf[i] = as_bf16x8(*(const uint4*)(q + at));
  }

  // loads: lane -> row of the load and chunk of it
  auto k_swizzle = [](int row) { return (row / (256 / RB)) & (CH - 1); };
  auto v_swizzle = [&](int row) { return I8 ? k_swizzle(row) : ((row / (256 / RB)) & (CH / 2 - 1)) * 2; };
  const int load_row = lane / CH, load_chunk_ = lane % CH;
  uint32_t k_off[LOADS], v_off[LOADS];
#pragma unroll
  for (int n = 0; n < LOADS; ++n) {
    const int row = n * PER + load_row;
    k_off[n] = row * RB + (load_chunk_ ^ k_swizzle(row)) * 16;
    v_off[n] = row * RB + (load_chunk_ ^ v_swizzle(row)) * 16;
  }
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_addr_of(lds) + wave * S * SLOT);
  // (through the scalar cache: a vector load here would be waited for, and with it all that are under way)
  typedef const __attribute__((address_space(4))) int* ScalarTable;
  const ScalarTable table = (ScalarTable)(uintptr_t)(g.seqs.pages + (long long)u.s * g.seqs.width);
  const int slot_mask = (1 << g.cache.page_shift) - 1;
  // the first of the 16 keys' rows, counted in rows of the cache
  auto group_row = [&](int key) {
    unsigned page = (unsigned)table[key >> g.cache.page_shift];
    page = page < g.cache.pages ? page : g.cache.pages - 1;
    return (((long long)page * g.cache.kv_heads + u.head) << g.cache.page_shift) + (key & slot_mask);
  };
  auto issue = [&](int block, int slot) {
    const uint32_t to = ring + slot * SLOT;
    long long base[2];
    int lo[2], hi[2];  // rows of the 16 that are loaded as they are
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      int key = block * KEYS + t * 16;
      const int k0 = low & ~15, k1 = high & ~15;
      key = key < k0 ? k0 : key > k1 ? k1 : key;
      base[t] = group_row(key);
      lo[t] = low - key > 0 ? low - key : 0;
      hi[t] = high - key < 15 ? high - key : 15;
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const unsigned char* from = uniform_pointer((kv ? g.cache.v : g.cache.k) + base[t] * RB);
#pragma unroll
        for (int n = 0; n < LOADS; ++n) {
          uint32_t off = kv ? v_off[n] : k_off[n];
          if (lo[t] > 0 || hi[t] < 15) {  // uniform
            const int row = n * PER + load_row;
            const int there = row < lo[t] ? lo[t] : row > hi[t] ? hi[t] : row;
            off += (there - row) * RB;
          }
          dma16_so(off, from, to + kv * TILE + (t * LOADS + n) * 1024);
        }
      }
    if (I8) {  // lane -> scale of a key (0..31) or a value (32..63)
      const int t = (lane >> 4) & 1, row = lane & 15;
      const int l0 = t ? lo[1] : lo[0], h0 = t ? hi[1] : hi[0];
      const int there = row < l0 ? l0 : row > h0 ? h0 : row;
      const float* from = (lane < 32 ? g.cache.k_scale : g.cache.v_scale) + (t ? base[1] : base[0]) + there;
      dma4(from, to + 2 * TILE);
    }
  };

  f32x4 oacc[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) oacc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float ref = kNothing, sum = 0.f;  // base 2; this lane's share of the sum

  const int mine = block1 - block0 > wave ? (block1 - block0 - wave + WAVES - 1) / WAVES : 0;
  if (mine > 0) issue(block0 + wave, 0);
  for (int i = 0; i < mine; ++i) {
    const int block = block0 + wave + i * WAVES, slot = i & 1;
    if (i + 1 < mine) {
      issue(block + WAVES, slot ^ 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COUNT) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    const unsigned char* ks = lds + wave * S * SLOT + slot * SLOT;
    const uint32_t vs = ring + slot * SLOT + TILE;
    f32x4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int row = t * 16 + r16;
#pragma unroll
      for (int i2 = 0; i2 < RB / 64; ++i2) {
        const uint4 w = *(const uint4*)(ks + row * RB + ((i2 * 4 + h) ^ k_swizzle(row)) * 16);
        if (I8) {
          const uint2 a = codes_to_bf16(w.x), b = codes_to_bf16(w.y), c = codes_to_bf16(w.z), d = codes_to_bf16(w.w);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(make_uint4(a.x, a.y, b.x, b.y)), qf[2 * i2], s[t], 0, 0, 0);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(make_uint4(c.x, c.y, d.x, d.y)), qf[2 * i2 + 1], s[t], 0, 0, 0);
        } else {
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), qf[i2], s[t], 0, 0, 0);
        }
      }
      if (I8) {
        const float4 sc = *(const float4*)(ks + 2 * TILE + (t * 16 + h * 4) * 4);
        s[t][0] *= sc.x * g.a2, s[t][1] *= sc.y * g.a2, s[t][2] *= sc.z * g.a2, s[t][3] *= sc.w * g.a2;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[t][e] *= g.a2;
      }
    }
    const int key0 = block * KEYS;
    // (a block that every row of the tile sees whole needs no mask; rows past the last see nothing and are not stored)
    const int least = u.seq.length - u.seq.n + u.tile * ROWS / g.group;
    const bool edge = key0 + KEYS - 1 > least || (g.window > 0 && key0 <= high - g.window);
    bool seen[2][4];
    if (edge) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = key0 + t * 16 + h * 4 + e;
          seen[t][e] = key <= pos && key >= first;
          if (!seen[t][e]) s[t][e] = -INFINITY;
        }
    }
    float top = ref;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = fmaxf(fmaxf(top, s[0][e]), s[1][e]);
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    if (__any(top > ref)) {
      const float back = __builtin_amdgcn_exp2f(ref - top);
      sum *= back;
#pragma unroll
      for (int x = 0; x < D / 16; ++x) oacc[x] *= back;
      ref = top;
    }
    float p[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[t][e] = __builtin_amdgcn_exp2f(s[t][e] - ref);
        sum += p[t][e];
      }
      if (I8) {
        const float4 sc = *(const float4*)(ks + 2 * TILE + 128 + (t * 16 + h * 4) * 4);
        p[t][0] *= sc.x, p[t][1] *= sc.y, p[t][2] *= sc.z, p[t][3] *= sc.w;
        if (edge) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!seen[t][e]) p[t][e] = 0.f;  // (its scale may be NaN)
        }
      }
    }
    const bf16x8 pf = as_bf16x8(make_uint4(pack_bf16x2(p[0][0], p[0][1]), pack_bf16x2(p[0][2], p[0][3]), pack_bf16x2(p[1][0], p[1][1]),
                                           pack_bf16x2(p[1][2], p[1][3])));
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      bf16x8 vf;
      if (I8) {
        const int k8 = (lane & 15) >> 1;  // of 8 keys: 4 h + (0..3), 16 + 4 h + (0..3)
        const int row = (k8 & 4) * 4 + h * 4 + (k8 & 3);
        const uint2 w = lds_read_tr8(vs + row * RB + (x ^ v_swizzle(row)) * 16 + (lane & 1) * 8);
        const uint2 a = codes_to_bf16(w.x), b = codes_to_bf16(w.y);
        vf = as_bf16x8(make_uint4(a.x, a.y, b.x, b.y));
      } else {
        const int i4 = lane & 15;
        const int row = h * 4 + (i4 >> 2);  // and 16 further: their swizzle is the same
        const uint32_t at = vs + row * RB + ((2 * x + ((i4 & 3) >> 1)) ^ v_swizzle(row)) * 16 + (i4 & 1) * 8;
        const uint2 a = lds_read_tr16(at), b = lds_read_tr16(at + 16 * RB);
        vf = as_bf16x8(make_uint4(a.x, a.y, b.x, b.y));
      }
      oacc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, oacc[x], 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the slot is refilled next)
  }
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);

  // the waves' sums [wave][row][D] meet in the ring's memory
  float* sums = (float*)lds;
  if (tid == 0) poisoned = 0;
  __syncthreads();
  if (h == 0) stat[wave][r16] = make_float2(ref, sum);
#pragma unroll
  for (int x = 0; x < D / 16; ++x)
    *(f32x4*)(sums + (wave * ROWS + r16) * D + (((x * 4 + h) ^ r16) * 4)) = oacc[x];  // (16-byte pieces spread over the banks)
  __syncthreads();
  constexpr int PIECES = ROWS * D / 4 / 256;
  float4 acc[PIECES];
  float2 mine_stat[PIECES];
  bool odd = false;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int at = i * 256 + tid, row = at / (D / 4), c = at % (D / 4);
    float top = kNothing;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, stat[w][row].x);
    float total = 0.f;
    acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float2 st = stat[w][row];
      const float back = __builtin_amdgcn_exp2f(st.x - top);
      const float4 v = *(const float4*)(sums + (w * ROWS + row) * D + ((c ^ row) * 4));
      total += st.y * back;
      acc[i].x += v.x * back, acc[i].y += v.y * back, acc[i].z += v.z * back, acc[i].w += v.w * back;
    }
    mine_stat[i] = make_float2(top, total);
    odd |= not_finite(acc[i].x) | not_finite(acc[i].y) | not_finite(acc[i].z) | not_finite(acc[i].w);
  }
  if (!I8) {
    if (__any(odd) && lane == 0) poisoned = 1;
    __syncthreads();
    if (poisoned) {
      for (int row = wave; row < ROWS; row += WAVES) {
        const int mm = u.tile * ROWS + row;
        if (mm < rows) careful_row<D>(g, u, mm, block0 * KEYS, block1 * KEYS, sums + row * D, (float*)&stat[0][row]);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int at = i * 256 + tid, row = at / (D / 4), c = at % (D / 4);
        acc[i] = *(const float4*)(sums + row * D + c * 4);
        mine_stat[i] = stat[0][row];
      }
    }
  }
  if (u.parts > 1 && u.part == 0 && tid == 0) {
    int* item = g.items + (1 + u.item) * kPagedItemWords;
    item[0] = u.slot, item[1] = u.parts, item[2] = u.tile, item[3] = u.head;
    item[4] = u.seq.first, item[5] = u.seq.n, item[6] = u.seq.length, item[7] = g.cache.kv_heads;  // (slots of a tile's parts are kv_heads apart)
  }
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int at = i * 256 + tid, row = at / (D / 4), c = at % (D / 4);
    const int mm = u.tile * ROWS + row;
    if (mm >= rows) continue;
    if (u.parts > 1) {
      const long long to = (long long)u.slot * ROWS + row;
      *(float4*)(g.part + to * D + c * 4) = acc[i];
      if (c == 0) g.stat[to] = mine_stat[i];
      continue;
    }
    const int tok = mm / g.group;
    const float inv = u.seq.length - u.seq.n + tok < 0 ? 0.f : 1.0f / mine_stat[i].y;
    u16* o = g.o + ((long long)(u.seq.first + tok) * g.heads + u.head * g.group + mm - tok * g.group) * D + c * 4;
    *(uint2*)o = make_uint2(pack_bf16x2(acc[i].x * inv, acc[i].y * inv), pack_bf16x2(acc[i].z * inv, acc[i].w * inv));
  }
}

// The parts of a tile joined: a workgroup a row, its waves sharing the parts.
template <int ROWS, int D>
__global__ void __launch_bounds__(256) paged_join_kernel(PagedArgs g) {
  __shared__ float2 wave_stat[4];
  __shared__ float wave_sums[4][D];
  const int item_i = blockIdx.x, row = blockIdx.y;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int* item = g.items + (1 + item_i) * kPagedItemWords;
  if (item_i >= g.items[0]) return;
  const int slot = item[0], parts = item[1], step = item[7], tile = item[2], mm = tile * ROWS + row;
  if (mm >= item[5] * g.group) return;
  constexpr int P = D / 64;
  float top = kNothing, total = 0.f, acc[P];
#pragma unroll
  for (int i = 0; i < P; ++i) acc[i] = 0.f;
  for (int x = wave; x < parts; x += 4) {
    const long long at = (long long)(slot + x * step) * ROWS + row;
    const float2 st = g.stat[at];
    float v[P];
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = g.part[at * D + i * 64 + lane];
    const float next = fmaxf(top, st.x), back = __builtin_amdgcn_exp2f(top - next), scale = __builtin_amdgcn_exp2f(st.x - next);
    total = total * back + st.y * scale;
#pragma unroll
    for (int i = 0; i < P; ++i) acc[i] = acc[i] * back + v[i] * scale;
    top = next;
  }
  if (lane == 0) wave_stat[wave] = make_float2(top, total);
#pragma unroll
  for (int i = 0; i < P; ++i) wave_sums[wave][i * 64 + lane] = acc[i];
  __syncthreads();
  if (threadIdx.x >= D) return;
  float t = kNothing, all = 0.f, y = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) t = fmaxf(t, wave_stat[w].x);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float scale = __builtin_amdgcn_exp2f(wave_stat[w].x - t);
    all += wave_stat[w].y * scale;
    y += wave_sums[w][threadIdx.x] * scale;
  }
  const int tok = mm / g.group;
  const float inv = item[6] - item[5] + tok < 0 ? 0.f : 1.0f / all;
  g.o[((long long)(item[4] + tok) * g.heads + item[3] * g.group + mm - tok * g.group) * D + threadIdx.x] = f2bf(y * inv);
}

}  // namespace nimble
#endif
