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
  Divisor by_group, by_heads;  // by `group`, by the heads of the cache
  int window;          // 0: none
  float a2;            // alpha log2 e
  float* part;         // [slots][rows][D] sums of parts, not divided
  float2* stat;        // [slots][rows] their largest score (base 2) and sum of probabilities
  int* items;          // [0]: tiles that may have been cut, then kPagedItemWords each, from the second entry on
  int slots, target_units, fewer_units;  // (fewer_units: see part_blocks)
  int step_shift;      // of the blocks of a step (SpanWalk)
  int once;            // keys and values are loaded past the caches
};

// (A division is some 25 instructions, 0.05 us where a workgroup begins, one behind the other.)
__device__ __forceinline__ int divided(int x, const Divisor& d) { return (int)(__umulhi(2u * (unsigned)x, d.magic) >> d.shift); }

constexpr float kNothing = -3.0e38f;  // the reference of a row that has seen no key yet

// ---------------------------------------------------------------------------
// What a workgroup does: a tile of ROWS rows of one sequence and one head of the cache, or a part of the keys that it sees.
// The rows of a (sequence, head) are its tokens times the query heads that share the head, row = token * group + query head: all of them
// meet the same keys.  Only the device knows the lengths, so it is the device that cuts: the key blocks of all tiles together, divided by
// the units that fill the chip, are what one part takes, and a tile that has more is cut into equal parts.  Every workgroup works
// this out for itself from all lengths, 64 sequences a step.  Heavy tiles of a sequence come first, the heads of the cache innermost: their
// workgroups go to the XCDs in turn, so that the tiles which read one head's keys share an L2.
// ---------------------------------------------------------------------------
struct PagedUnit {
  Sequence seq;
  int s, head, tile, tiles;  // tiles: of the sequence (SpanWalk only)
  int part, parts;
  int slot, item;  // in the workspace; slot -1: the tile was not cut
};

// Inclusive sums over the 64 lanes, in registers.
template <typename T>
__device__ __forceinline__ T wave_scan(T x) {
  auto step = [&](auto ctrl, auto rows) {
    constexpr int C = decltype(ctrl)::value, R = decltype(rows)::value;
    unsigned w[sizeof(T) / 4];
    __builtin_memcpy(w, &x, sizeof x);
#pragma unroll
    for (unsigned& y : w) y = (unsigned)__builtin_amdgcn_update_dpp(0, (int)y, C, R, 0xf, false);
    T y;
    __builtin_memcpy(&y, w, sizeof y);
    x += y;
  };
  using std::integral_constant;
  step(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});  // from 1, 2, 4 and 8 lanes below in a row of 16
  step(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});  // the last of rows 0 and 2 to rows 1 and 3
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});  // the last of row 1 to rows 2 and 3
  return x;
}

__device__ __forceinline__ int wave_max(int x) {  // of values from 0 on
  auto step = [&](auto ctrl, auto rows) {
    const int y = __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    x = y > x ? y : x;
  };
  using std::integral_constant;
  step(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
  return __builtin_amdgcn_readlane(x, 63);
}

template <int ROWS, int KEYS>
__device__ __forceinline__ void tile_work(const PagedArgs& g, const Sequence& q, int& tiles, int& blocks) {
  tiles = (q.n * g.group + ROWS - 1) / ROWS;  // (at most 2^24 rows of 2^6 heads and so on: checked by the host)
  int keys = q.length;
  if (g.window > 0 && g.window + ROWS < keys) keys = g.window + ROWS;
  blocks = tiles ? (keys + KEYS - 1) / KEYS : 0;
}

// The blocks of one part, give or take half as many: a tile is cut into as many parts as comes closest, since what is left of one that is a little too
// long costs a part's prologue and a join.  Fewer units where parts of as many as fit would be of less than 16 blocks (heads of 64, of which a compute unit holds
// three and not two: 2048 rows over 16384 keys, 16 heads of 64 in bf16, 150 us with two to a compute unit, 136 with three, in 8 bits 231 and 196; 128 rows over
// 30128 keys, 10 blocks a part, 36.9 and 40.2).  The same in every lane of every wave of a call.
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
  total = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_scan(total)), 63));
  total *= (float)g.cache.kv_heads;
  float most = total / (float)g.target_units;
  if (most < 16.0f) most = total / (float)g.fewer_units;
  most = ceilf(most) + 1.0f;
  return most < (float)LEAST ? LEAST : most > 1.0e9f ? 1000000000 : (int)most;
}

// One wave finds the workgroup's unit (four at once take four times as long) and leaves it in `shared`, kUnitWords words of LDS; behind a barrier
// take_unit reads it, and the number of tiles that are cut (the last word, where unit = 0).
constexpr int kUnitWords = 12;
template <int ROWS, int KEYS, int LEAST>
__device__ __forceinline__ void find_unit(const PagedArgs& g, unsigned unit, int* shared) {
  const int lane = threadIdx.x & 63, G = g.cache.kv_heads;
  const int most = g.slots ? part_blocks<ROWS, KEYS, LEAST>(g) : 1000000000;
  const unsigned want = (unsigned)divided((int)unit, g.by_heads);
  const int head = (int)(unit - want * G);
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
    int parts = 1;
    unsigned b = 0, c = 0;
    if (g.slots) {
      const unsigned p = ((unsigned)blocks + (unsigned)most / 2) / (unsigned)most;
      parts = p > 1 ? (int)p : 1;
    }
    const unsigned mine = (unsigned)tiles * parts, mine_cut = parts > 1 ? mine : 0, tiles_cut = parts > 1 ? tiles : 0;
    if (g.slots) b = wave_scan(mine_cut), c = wave_scan(tiles_cut);
    // of these 64 sequences the long ones first, in four classes: what begins last should not take longest
    const int longest = wave_max(blocks);
    unsigned start = units;
#pragma unroll
    for (int k = 3; k >= 0; --k) {
      const bool in = (k == 0 || blocks * 4ll > (long long)longest * k) && (k == 3 || blocks * 4ll <= (long long)longest * (k + 1));
      const unsigned upto = wave_scan(in ? mine : 0u);
      if (in) start = units + upto - mine;
      units += (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
    }
    const bool here = mine > 0 && want >= start && want - start < mine;
    if (!found && __any(here)) {
      found = true;
      if (here) {
        const int rest = (int)(want - start), back = parts == 1 ? rest : rest / parts;
        shared[0] = 1;
        shared[1] = s;
        shared[2] = q.first;
        shared[3] = q.n;
        shared[4] = q.length;
        shared[5] = tiles - 1 - back;
        shared[6] = rest - back * parts;
        shared[7] = parts;
        shared[8] = parts == 1 ? -1 : (int)((cut_units + b - mine_cut + rest) * G + head);
        shared[9] = (int)((cut_tiles + c - tiles_cut + back) * G + head);
        shared[10] = head;
      }
    }
    if (g.slots) {
      cut_units += (unsigned)__builtin_amdgcn_readlane((int)b, 63);
      cut_tiles += (unsigned)__builtin_amdgcn_readlane((int)c, 63);
    }
  }
  if (lane == 0) {
    if (!found) shared[0] = 0;
    shared[11] = (int)cut_tiles * G;
  }
}
__device__ __forceinline__ bool take_unit(const int* shared, PagedUnit& u) {
  auto word = [&](int i) { return __builtin_amdgcn_readfirstlane(shared[i]); };
  u.s = word(1);
  u.seq = Sequence{word(2), word(3), word(4)};
  u.tile = word(5);
  u.part = word(6);
  u.parts = word(7);
  u.slot = word(8);
  u.item = word(9);
  u.head = word(10);
  return word(0) != 0;
}

// The keys of a tile, and of one part of it, in blocks.
template <int ROWS, int KEYS>
__device__ __forceinline__ void unit_keys(const PagedArgs& g, const PagedUnit& u, int& low, int& high, int& block0, int& block1) {
  const int m0 = u.tile * ROWS, rows = u.seq.n * g.group, m1 = (m0 + ROWS < rows ? m0 + ROWS : rows) - 1;
  const int before = u.seq.length - u.seq.n;
  high = before + divided(m1, g.by_group);                                             // the last key that a row of the tile sees
  low = 0;
  if (g.window > 0) {
    low = before + divided(m0, g.by_group) - g.window + 1;                             // and the first
    if (low < 0) low = 0;
  }
  low = __builtin_amdgcn_readfirstlane(low);
  high = __builtin_amdgcn_readfirstlane(high);
  if (high < 0) {
    block0 = block1 = 0;
    return;
  }
  const int b0 = low / KEYS, nb = high / KEYS + 1 - b0;
  if (u.parts == 1) {
    block0 = b0;
    block1 = b0 + nb;
    return;
  }
  const int q = nb / u.parts, r = nb - q * u.parts;  // (the first r parts have one more)
  block0 = __builtin_amdgcn_readfirstlane(b0 + u.part * q + (u.part < r ? u.part : r));
  block1 = __builtin_amdgcn_readfirstlane(block0 + q + (u.part < r ? 1 : 0));
}

// ---------------------------------------------------------------------------
// The other way to share the work, for few rows, where a tile is one sequence's keys and what counts is that every workgroup has the same
// number of them: the blocks of all tiles in a row, one sequence after the other, cut into spans of equal length, one a workgroup.  A span may
// end one tile, hold several and begin another.  A workgroup leaves at most two parts: of the tile that another one began (slot 2 w) and of
// the one that it begins (slot 2 w + 1); the second launch finds a cut tile by the workgroup that began it.
//   Lengths are counted in steps of 2^step_shift blocks, a tile as many as the longest of its sequence; a share of them is that share of the blocks that
// the tile has.  (64 sequences of up to 8192 keys, uneven, as tiles cut into equal parts of at most a 512th of all: 144 us, 1.5 rounds
// of workgroups; in spans 121.)
// ---------------------------------------------------------------------------
template <int ROWS, int KEYS, bool CUT>
struct SpanWalk {
  const PagedArgs& g;
  int base;                // this lane's sequence is base + lane
  Sequence q;
  int tiles, steps;
  unsigned ahead, upto;    // steps of the sequences ahead of these 64, and up to this lane's with them
  unsigned at, end, per;   // what is left of the span, and its length
  bool none;               // the span is empty

  static __device__ __forceinline__ unsigned lane_value(unsigned x, int l) { return (unsigned)__builtin_amdgcn_readlane((int)x, l); }
  __device__ __forceinline__ unsigned look(int s) {
    q = Sequence{0, 0, 0};
    tiles = steps = 0;
    if (s >= g.seqs.count) return 0;
    q = sequence_of(g.seqs, s, g.cache.page_shift);
    int blocks;
    tile_work<ROWS, KEYS>(g, q, tiles, blocks);
    steps = CUT ? (blocks + (1 << g.step_shift) - 1) >> g.step_shift : 0;
    if (steps == 0) steps = tiles > 0;  // rows that see nothing; without a workspace a tile is a step and so is a span
    return (unsigned)tiles * (unsigned)steps * (unsigned)g.cache.kv_heads;  // (all of them fewer than 2^31: checked by the host)
  }
  __device__ __forceinline__ void load(int b) {
    base = b;
    upto = ahead + wave_scan(look(b + (threadIdx.x & 63)));
  }
  __device__ __forceinline__ SpanWalk(const PagedArgs& args, unsigned w) : g(args) {
    unsigned total = 0;
    ahead = 0;
    if (g.seqs.count > 64) {
      for (int b = 0; b < g.seqs.count; b += 64) total += look(b + (threadIdx.x & 63));
      total = lane_value(wave_scan(total), 63);
      load(0);
    } else {
      load(0);
      total = lane_value(upto, 63);
    }
    per = CUT ? (total + (unsigned)g.target_units - 1) / (unsigned)g.target_units : 1;
    if (per == 0) per = 1;
    const unsigned long long from = (unsigned long long)w * per;
    none = from >= total;
    at = none ? total : (unsigned)from;
    end = total - at < per ? total : at + per;
  }
  // The tile that the rest of the span begins with: steps x0 .. x1 - 1 of its u.parts.  tile_at: where the tile begins.
  __device__ __forceinline__ void next(PagedUnit& u, unsigned& x0, unsigned& x1, unsigned& tile_at) {
    while (at >= lane_value(upto, 63)) {
      ahead = lane_value(upto, 63);
      load(base + 64);
    }
    const int l = __ffsll(__ballot(upto > at)) - 1;
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
    u.s = base + l;
    u.seq.first = of(q.first);
    u.seq.n = of(q.n);
    u.seq.length = of(q.length);
    u.tiles = of(tiles);
    u.parts = CUT ? of(steps) : 1;
    const unsigned G = (unsigned)g.cache.kv_heads;
    const unsigned first = lane_value(upto, l) - (unsigned)u.tiles * (unsigned)u.parts * G;
    const unsigned which = u.parts == 1 ? at - first : (at - first) / (unsigned)u.parts;
    tile_at = first + which * (unsigned)u.parts;
    u.tile = divided((int)which, g.by_heads);
    u.head = (int)(which - (unsigned)u.tile * G);
    x0 = at - tile_at;
    x1 = end - tile_at < (unsigned)u.parts ? end - tile_at : (unsigned)u.parts;
    at = tile_at + x1;
  }
  // The workgroup whose span holds step x.
  __device__ __forceinline__ unsigned owner(unsigned x) const { return x / per; }
};

// The blocks of a span's share of a tile.
template <int ROWS, int KEYS>
__device__ __forceinline__ void share_keys(const PagedArgs& g, const PagedUnit& u, unsigned x0, unsigned x1, int& low, int& high, int& block0, int& block1) {
  PagedUnit all = u;
  all.part = 0;
  all.parts = 1;
  unit_keys<ROWS, KEYS>(g, all, low, high, block0, block1);
  if (x0 == 0 && x1 == (unsigned)u.parts) return;
  const unsigned nb = block1 - block0;                      // below 2^26, and steps below 2^23
  const unsigned q = nb / (unsigned)u.parts, r = nb - q * (unsigned)u.parts;   // (the first r steps have one block more)
  const int b0 = block0;
  block0 = __builtin_amdgcn_readfirstlane(b0 + (int)(x0 * q + (x0 < r ? x0 : r)));
  block1 = __builtin_amdgcn_readfirstlane(b0 + (int)(x1 * q + (x1 < r ? x1 : r)));
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

// What the second launch has to know of a tile that was cut: its first part's slot, the second's, and how far apart those behind it are.
__device__ __forceinline__ void put_item(const PagedArgs& g, const PagedUnit& u, int which, int parts, int slot, int second, int apart) {
  int* item = g.items + (1 + which) * kPagedItemWords;
  item[0] = parts, item[1] = slot, item[2] = second, item[3] = apart;
  item[4] = u.tile, item[5] = u.head, item[6] = u.seq.first, item[7] = u.seq.n, item[8] = u.seq.length;
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
