// Attention of few rows over a paged cache.
#ifndef NIMBLE_PAGED_TOKENS_KERNEL_H_
#define NIMBLE_PAGED_TOKENS_KERNEL_H_
#include "paged_common.h"

namespace nimble {

// ---------------------------------------------------------------------------
// Few rows: 16 of a (sequence, head) per workgroup, WAVES waves that each take every WAVES-th block of 32 keys and meet at the end.
//   scores:  MFMA 16x16x32, 16 keys on the A side, the 16 rows on the B side: lane (r, h) = (lane & 15, lane >> 4) holds, for row r, keys
//            16 t + 4 h + (0..3) of tile t = 0, 1.
//   P.V:     the 8 k slots of h are defined as the keys it holds, 4 of either tile, so that P stays in its lane; the values come out of
//            the row-major tile with the transposing LDS read (of 16 bits a piece, or of 8).
//   8 bits:  codes become bf16, which holds them exactly, behind the LDS reads; a key's scale multiplies its scores, a value's its
//            probability.  A lane reads 16 codes of a key row where it reads 8 elements of bf16, so that the elements of a
//            matrix instruction's k are taken from the row in another order, and those of q in the same.
//   Work:    a workgroup walks its span of all tiles' blocks (SpanWalk); without CUT it has one tile (what is left out ahead of the loop and behind it: one token
//            over 777 keys 7.55 -> 6.9 us, chunks of 77 rows 12.6 -> 12.0).
//   Loads:   direct global->LDS loads into the wave's own ring of two blocks, waited for by count: no barrier in the loop.  16 keys lie in one
//            page, whose number is a scalar.  Chunk c of row r sits at c ^ swizzle(r).  Keys outside of what the tile sees repeat the
//            nearest one that it does.
//   Bound by memory where the cache is large: one token over 131001 keys, 8 heads of 128 in bf16, 87.4 us, 537 MB at 6.1 TB/s, of which 5.1 are the second
// launch (a kernel that only reads reaches 6.4 to 6.5); 64 tokens over up to 8192 keys in 8 bits 99 us, 563 MB at 5.7 TB/s: two tiles a workgroup, whose
// beginnings and ends nothing hides.  One token over 777 keys, 16 heads of 64: 6.9 us, a launch, three loads one behind the other for the unit,
// the wave's three blocks and the meeting of eight waves.
// ---------------------------------------------------------------------------
// (As many waves a SIMD as the LDS holds: with fewer the spans, one for each, go in two rounds.  64 tokens over 4096 keys, 16 heads of 64 in 8 bits, with three
// of four 121 us, 100.  Told so the compiler also orders heads of 128 better: 64 tokens over up to 8192 keys 106.3 -> 101.0 us.)
template <int D, bool I8, int WAVES, bool CUT>
__global__ void __launch_bounds__(WAVES * 64) __attribute__((amdgpu_waves_per_eu((D == 64 ? 2 : 1) * (I8 ? 2 : 1)))) paged_tokens_kernel(PagedArgs g) {
  constexpr int ROWS = 16, KEYS = kPagedBlockKeys, T = WAVES * 64;
  constexpr int RB = D * (I8 ? 1 : 2);           // bytes of a key row
  constexpr int CH = RB / 16;                    // its chunks
  constexpr int PER = 1024 / RB;                 // rows of one load
  constexpr int LOADS = 16 / PER;                // loads of 16 rows
  constexpr int TILE = KEYS * RB;                // bytes of a block of K or V
  constexpr int SCALES = I8 ? 256 : 0;           // 32 scales of keys, 32 of values
  constexpr int SLOT = 2 * TILE + SCALES;
  constexpr int S = 2;
  constexpr int KL = 2 * LOADS + (I8 ? 1 : 0), VL = 2 * LOADS;  // loads of a block's keys (with the scales of both), of its values
  constexpr int RING = WAVES * S * SLOT, JOIN = WAVES * ROWS * D * 4;
  __shared__ __attribute__((aligned(256))) unsigned char lds[RING > JOIN ? RING : JOIN];
  __shared__ float2 stat[WAVES][ROWS];
  __shared__ int poisoned;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, h = lane >> 4;
  SpanWalk<ROWS, KEYS, CUT> walk(g, blockIdx.x);
  walk.clear_item();
  if (walk.none) return;
  for (bool again = true; again; again = CUT && walk.at < walk.end) {
  PagedUnit u;
  int low, high, block0, block1;
  walk.take(u, low, high, block0, block1);

  // this lane's row
  const int m = u.tile * ROWS + r16, rows = u.seq.n * g.group;
  const int m_ld = m < rows ? m : rows - 1;
  const int token = divided(m_ld, g.by_group);
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
  const int* table = g.seqs.pages + (long long)u.s * g.seqs.width;
  const int slot_mask = (1 << g.cache.page_shift) - 1;
  const int k0 = low & ~15, k1 = high & ~15;
  auto held_to = [&](int key) { return key < k0 ? k0 : key > k1 ? k1 : key; };
  // The pages of the wave's next 64 blocks: lane l holds that of keys 16 (l & 1) .. + 15 of its blocks l / 2 and 32 + l / 2.  (Looked up block by block
  // through the scalar cache a block of a wave took 0.77 us of one token over 777 keys of 64, most of it waiting for its page.)
  int pages0 = 0, pages1 = 0;
  auto page_at = [&](int i) { return table[held_to((block0 + wave + i * WAVES) * KEYS + (lane & 1) * 16) >> g.cache.page_shift]; };
  auto look_up = [&](int first) {  // from the wave's block `first` on
    pages0 = page_at(first + (lane >> 1));
    pages1 = page_at(first + 32 + (lane >> 1));
  };
  // the first of 16 keys' rows, counted in rows of the cache
  auto group_row = [&](int i, int t, int key) {
    unsigned page = (unsigned)__builtin_amdgcn_readlane(i & 32 ? pages1 : pages0, (i & 31) * 2 + t);
    page = page < g.cache.pages ? page : g.cache.pages - 1;
    return (((long long)page * g.cache.kv_heads + u.head) << g.cache.page_shift) + (key & slot_mask);
  };
  // Where a block's two times 16 keys are: rows of the cache, and whether all are loaded as they are.
  struct Place {
    long long row[2];
    int key[2];
    bool whole;
  };
  auto place_of = [&](int i) {  // of the wave's block i
    if (i && (i & 63) == 0) look_up(i);
    const int key0 = (block0 + wave + i * WAVES) * KEYS;
    Place p;
    p.whole = key0 >= low && key0 + KEYS - 1 <= high;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      p.key[t] = held_to(key0 + t * 16);
      p.row[t] = group_row(i, t, p.key[t]);
    }
    return p;
  };
  // (One branch for all of a block's loads, and one for their kind: with one or two for each load they took half of the loop's instructions; one token
  // over 777 keys 8.4 -> 7.5 us, 64 over up to 8192 in 8 bits 100.7 -> 98.8, chunks of 77 rows 13.4 -> 12.7.)
  auto issue = [&](auto is_v, const Place& p, int slot) {
    constexpr bool V = decltype(is_v)::value;
    const uint32_t to = ring + slot * SLOT + V * TILE;
    const unsigned char* from[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) from[t] = uniform_pointer((V ? g.cache.v : g.cache.k) + p.row[t] * RB);
    auto nearest = [&](int t, int row) {  // the row that stands in for one of the 16
      const int lo = low - p.key[t] > 0 ? low - p.key[t] : 0, hi = high - p.key[t] < 15 ? high - p.key[t] : 15;
      return row < lo ? lo : row > hi ? hi : row;
    };
    if (!p.whole) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < LOADS; ++n) {
          const int row = n * PER + load_row;
          dma16_so((V ? v_off[n] : k_off[n]) + (uint32_t)((nearest(t, row) - row) * RB), from[t], to + (t * LOADS + n) * 1024);
        }
    } else if (g.once) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < LOADS; ++n) dma16_so_once(V ? v_off[n] : k_off[n], from[t], to + (t * LOADS + n) * 1024);
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < LOADS; ++n) dma16_so(V ? v_off[n] : k_off[n], from[t], to + (t * LOADS + n) * 1024);
    }
    if (I8 && !V) {  // lane -> scale of a key (0..31) or a value (32..63)
      const int t = (lane >> 4) & 1;
      const int row0 = p.whole ? lane & 15 : nearest(0, lane & 15), row1 = p.whole ? lane & 15 : nearest(1, lane & 15);
      const long long at0 = p.row[0] + row0, at1 = p.row[1] + row1;
      dma4((lane < 32 ? g.cache.k_scale : g.cache.v_scale) + (t ? at1 : at0), to + 2 * TILE);
    }
  };
  using K_TILE = std::false_type;
  using V_TILE = std::true_type;

  f32x4 oacc[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) oacc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float ref = kNothing, sum = 0.f;  // in units of the scores; this lane's share of the sum

  const int mine = block1 - block0 > wave ? (block1 - block0 - wave + WAVES - 1) / WAVES : 0;
  // Three halves of a block are under way beside the one in work: the values of block i + 1 are asked for ahead of block i's scores, the keys of
  // block i + 2 behind them, when those of block i have been read.
  Place next{};
  if (mine > 0) {
    look_up(0);
    const Place p = place_of(0);
    issue(K_TILE{}, p, 0);
    issue(V_TILE{}, p, 0);
    if (mine > 1) {
      next = place_of(1);
      issue(K_TILE{}, next, 1);
    }
  }
  for (int i = 0; i < mine; ++i) {
    const int block = block0 + wave + i * WAVES, slot = i & 1;
    if (i + 1 < mine) {
      issue(V_TILE{}, next, slot ^ 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(KL + 2 * VL) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(VL) : "memory");
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
        s[t][0] *= sc.x, s[t][1] *= sc.y, s[t][2] *= sc.z, s[t][3] *= sc.w;
      }
    }
    f32x4 v_scale[2];
    if (I8) {
#pragma unroll
      for (int t = 0; t < 2; ++t) v_scale[t] = *(const f32x4*)(ks + 2 * TILE + 128 + (t * 16 + h * 4) * 4);
    }
    if (i + 2 < mine) {
      next = place_of(i + 2);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the keys and the scales have been read)
      issue(K_TILE{}, next, slot);
    }
    if (i + 2 < mine)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * KL + VL) : "memory");
    else if (i + 1 < mine)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(KL + VL) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // The values are read out of LDS ahead of the softmax, behind which their way would be waited for: one token over 777 keys 8.9 -> 8.7 us, 64 over up
    // to 8192 in 8 bits 108.9 -> 107.5.
    uint2 va[D / 16], vb[I8 ? 1 : D / 16];
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      if (I8) {
        const int k8 = (lane & 15) >> 1;  // of 8 keys: 4 h + (0..3), 16 + 4 h + (0..3)
        const int row = (k8 & 4) * 4 + h * 4 + (k8 & 3);
        va[x] = lds_read_tr8(vs + row * RB + (x ^ v_swizzle(row)) * 16 + (lane & 1) * 8);
      } else {
        const int i4 = lane & 15;
        const int row = h * 4 + (i4 >> 2);  // and 16 further: their swizzle is the same
        const uint32_t at = vs + row * RB + ((2 * x + ((i4 & 3) >> 1)) ^ v_swizzle(row)) * 16 + (i4 & 1) * 8;
        va[x] = lds_read_tr16(at), vb[x] = lds_read_tr16(at + 16 * RB);
      }
    }
    const int key0 = block * KEYS;
    // (a block that every row of the tile sees whole needs no mask; rows past the last see nothing and are not stored)
    const int least = u.seq.length - u.seq.n + divided(u.tile * ROWS, g.by_group);
    const bool edge = key0 + KEYS - 1 > least || (g.window > 0 && key0 <= high - g.window);
    if (edge) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = key0 + t * 16 + h * 4 + e;
          if (key <= pos && key >= first) continue;
          s[t][e] = -INFINITY;
          if (I8) v_scale[t][e] = 0.f;  // (it may be NaN)
        }
    }
    float top = ref;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = fmaxf(fmaxf(top, s[0][e]), s[1][e]);
    {  // of the row's four quarters
      const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
      const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    if (__any(top > ref)) {
      const float back = __builtin_amdgcn_exp2f((ref - top) * g.a2);
      sum *= back;
#pragma unroll
      for (int x = 0; x < D / 16; ++x) oacc[x] *= back;
      ref = top;
    }
    const float nm2 = ref > kNothing ? -ref * g.a2 : 0.f;  // (a row that has seen nothing: its scores are minus infinity)
    float p[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[t][e] = __builtin_amdgcn_exp2f(fmaf(s[t][e], g.a2, nm2));
        sum += p[t][e];
        if (I8) p[t][e] *= v_scale[t][e];
      }
    }
    // The probabilities in two bf16, what the first leaves of them in the second: 2^-16 of each is lost at most, where one would lose 2^-8, as much
    // as the rounding of the result does (relative to it 0.0017 in all, with one 0.0020 to 0.0025).  It costs little where loads are what is waited for:
    // one token over 131001 keys 86.9 -> 87.8 us, 64 over up to 8192 in 8 bits 105.7 -> 108.7, one over 777 8.7 -> 8.9.
    uint32_t ph[4], pl[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float p0 = p[x >> 1][(x & 1) * 2], p1 = p[x >> 1][(x & 1) * 2 + 1];
      ph[x] = pack_bf16x2(p0, p1);
      pl[x] = pack_bf16x2(p0 - of_pair(ph[x], 0), p1 - of_pair(ph[x], 1));
    }
    const bf16x8 pf = as_bf16x8(make_uint4(ph[0], ph[1], ph[2], ph[3])), pf_low = as_bf16x8(make_uint4(pl[0], pl[1], pl[2], pl[3]));
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      bf16x8 vf;
      if (I8) {
        const uint2 a = codes_to_bf16(va[x].x), b = codes_to_bf16(va[x].y);
        vf = as_bf16x8(make_uint4(a.x, a.y, b.x, b.y));
      } else {
        vf = as_bf16x8(make_uint4(va[x].x, va[x].y, vb[I8 ? 0 : x].x, vb[I8 ? 0 : x].y));
      }
      oacc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, oacc[x], 0, 0, 0);
      oacc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf_low, oacc[x], 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the values' slot is refilled next)
  }
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);

  // the waves' sums [wave][row][D] meet in the ring's memory
  float* sums = (float*)lds;
  if (tid == 0) poisoned = 0;
  __syncthreads();
  if (h == 0) stat[wave][r16] = make_float2(ref > kNothing ? ref * g.a2 : kNothing, sum);
#pragma unroll
  for (int x = 0; x < D / 16; ++x)
    *(f32x4*)(sums + (wave * ROWS + r16) * D + (((x * 4 + h) ^ r16) * 4)) = oacc[x];  // (16-byte pieces spread over the banks)
  __syncthreads();
  constexpr int PIECES = (ROWS * D / 4 + T - 1) / T;
  float4 acc[PIECES];
  float2 mine_stat[PIECES];
  bool odd = false;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int at = i * T + tid, row = at / (D / 4) % ROWS, c = at % (D / 4);
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
  bool careful = false;
  if (!I8) {
    if (__any(odd) && lane == 0) poisoned = 1;
    __syncthreads();
    careful = poisoned;
  }
  if (careful) {
    for (int row = wave; row < ROWS; row += WAVES)
      if (u.tile * ROWS + row < rows) careful_row<ROWS, D>(g, u, u.tile * ROWS + row, block0 * KEYS, block1 * KEYS);
  } else {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int at = i * T + tid, row = at / (D / 4), c = at % (D / 4);
      const int mm = u.tile * ROWS + row;
      if (row >= ROWS || mm >= rows) continue;
      if (u.slot >= 0) {
        const long long to = (long long)u.slot * ROWS + row;
        *(float4*)(g.part + to * D + c * 4) = acc[i];
        if (c == 0) g.stat[to] = mine_stat[i];
        continue;
      }
      const int tok = divided(mm, g.by_group);
      const float inv = u.seq.length - u.seq.n + tok < 0 ? 0.f : 1.0f / mine_stat[i].y;
      u16* o = g.o + ((long long)(u.seq.first + tok) * g.heads + u.head * g.group + mm - tok * g.group) * D + c * 4;
      *(uint2*)o = make_uint2(pack_bf16x2(acc[i].x * inv, acc[i].y * inv), pack_bf16x2(acc[i].z * inv, acc[i].w * inv));
    }
  }
  __syncthreads();  // (the ring is filled again)
  }
}

}  // namespace nimble
#endif
