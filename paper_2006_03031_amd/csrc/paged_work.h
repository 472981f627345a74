// Attention of new rows over a paged cache: what each workgroup does, and how long sequences are cut into parts.  (Integers, offsets and
// lengths only: tests/paged_work_cpu.cpp builds this file for the CPU, lane by lane.)
#ifndef NIMBLE_PAGED_WORK_H_
#define NIMBLE_PAGED_WORK_H_
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

// What the second launch has to know of a tile that was cut: its first part's slot, the second's, and how far apart those behind it are.
__device__ __forceinline__ void put_item(const PagedArgs& g, const PagedUnit& u, int which, int parts, int slot, int second, int apart) {
  int* item = g.items + (1 + which) * kPagedItemWords;
  item[0] = parts, item[1] = slot, item[2] = second, item[3] = apart;
  item[4] = u.tile, item[5] = u.head, item[6] = u.seq.first, item[7] = u.seq.n, item[8] = u.seq.length;
}
// Behind a unit of find_unit: by its first part.
__device__ __forceinline__ void put_unit_item(const PagedArgs& g, const PagedUnit& u) {
  if (u.parts > 1 && u.part == 0 && threadIdx.x == 0) put_item(g, u, u.item, u.parts, u.slot, u.slot + g.cache.kv_heads, g.cache.kv_heads);
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
      if (units > 1u << 30) units = 1u << 30;  // (only with offsets that fall; 64 sequences have fewer than 2^30)
    }
  }
  // Offsets that fall give more units than the grid has workgroups.  Then there is nothing to join: parts of some tiles are computed by nobody.
  if (g.slots && unit == 0 && units > (unsigned)divided((int)gridDim.x, g.by_heads)) cut_tiles = 0;
  if (lane == 0) {
    if (!found) shared[0] = 0;
    shared[11] = (int)cut_tiles * G;
  }
}
__device__ __forceinline__ bool take_unit(const PagedArgs& g, const int* shared, PagedUnit& u) {
  auto word = [&](int i) { return __builtin_amdgcn_readfirstlane(shared[i]); };
  u.s = word(1);
  u.seq = Sequence{word(2), word(3), word(4)};
  u.tile = word(5);
  u.part = word(6);
  u.parts = word(7);
  u.slot = word(8);
  u.item = word(9);
  u.head = word(10);
  const bool found = word(0) != 0;
  if (g.slots && blockIdx.x == 0 && threadIdx.x == 0) g.items[0] = shared[11];
  return found && !(u.parts > 1 && (u.slot >= g.slots || u.item >= g.target_units));  // (not with offsets that keep to their description)
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

// ---------------------------------------------------------------------------
// The other way to share the work, for few rows, where a tile is one sequence's keys and what counts is that every workgroup has the same
// number of them: the blocks of all tiles in a row, one sequence after the other, cut into spans of equal length, one a workgroup.  A span may
// end one tile, hold several and begin another.  A workgroup leaves at most two parts: of the tile that another one began (slot 2 w) and of
// the one that it begins (slot 2 w + 1); the second launch finds a cut tile by the workgroup that began it.
//   Sequences that share rows (offsets that fall) may have steps that pass 32 bits together.  A tile that the walk takes is one of its sequence all the same: the
// sums ahead of it are not past `at`, the sum with it is, and one sequence has fewer than 2^31 steps, so that its own did not wrap.  But it may end behind
// the last span, whose parts nobody has; then it is not joined.
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
    return (unsigned)tiles * (unsigned)steps * (unsigned)g.cache.kv_heads;  // (fewer than 2^31, of one sequence or of all: checked by the host)
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
  // Ahead of the span: an entry for the second launch that says that nothing was cut here.
  __device__ __forceinline__ void clear_item() const {
    if (!CUT || threadIdx.x != 0) return;
    if (blockIdx.x == 0) g.items[0] = (int)gridDim.x;
    g.items[(1 + blockIdx.x) * kPagedItemWords] = 0;
  }
  // The tile that the rest of the span begins with, and the blocks of it that are this workgroup's.
  __device__ __forceinline__ void take(PagedUnit& u, int& low, int& high, int& block0, int& block1) {
    unsigned x0, x1, tile_at;
    next(u, x0, x1, tile_at);
    u.slot = !CUT || (x0 == 0 && x1 == (unsigned)u.parts) ? -1 : 2 * (int)blockIdx.x + (x0 == 0);
    if (CUT) {
      share_keys<ROWS, KEYS>(g, u, x0, x1, low, high, block0, block1);
    } else {
      u.part = 0;
      unit_keys<ROWS, KEYS>(g, u, low, high, block0, block1);
    }
    if (CUT && x0 == 0 && x1 < (unsigned)u.parts && threadIdx.x == 0) {
      const unsigned last = owner(tile_at + u.parts - 1);
      if (last < gridDim.x) put_item(g, u, (int)blockIdx.x, (int)last - (int)blockIdx.x + 1, u.slot, 2 * ((int)blockIdx.x + 1), 2);
    }
  }
};

// What of a call's arguments follows from its extents and its plan.
inline void set_extents(PagedArgs& g, const nimble_cache& c, const nimble_sequences& s, int64_t heads, int64_t window) {
  g.cache = cache_args(c);
  g.seqs = sequences_args(s);
  if (c.pages == 0) g.seqs.width = 0;  // nothing is cached
  g.heads = (int)heads;
  g.group = (int)(heads / c.kv_heads);
  g.by_group = divisor_of(g.group);
  g.by_heads = divisor_of(c.kv_heads);
  g.window = (int)(window < kMostPositions ? window : 0);  // (2^30 and beyond: all)
}
inline void set_parts(PagedArgs& g, const nimble_paged_plan& p, int64_t D, void* workspace) {
  if (!p.parts) return;
  g.slots = (int)p.slots;
  g.target_units = (int)(p.slots - 8) / 2;  // (see plan_paged)
  while ((kPagedBlockKeys << g.step_shift) < p.step) ++g.step_shift;
  g.fewer_units = g.target_units < 2 * kComputeUnits ? g.target_units : 2 * kComputeUnits;
  g.part = (float*)workspace;
  g.stat = (float2*)(g.part + p.slots * p.rows * D);
  g.items = (int*)(g.stat + p.slots * p.rows);
}

}  // namespace nimble
#endif
