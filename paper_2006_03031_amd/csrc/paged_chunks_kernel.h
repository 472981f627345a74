// Attention of many rows over a paged cache.
#ifndef NIMBLE_PAGED_CHUNKS_KERNEL_H_
#define NIMBLE_PAGED_CHUNKS_KERNEL_H_
#include "paged_common.h"

namespace nimble {

// ---------------------------------------------------------------------------
// Many rows: 128 of a (sequence, head) per workgroup, 32 a wave, all over the same blocks of 64 keys.
//   scores:  MFMA 32x32x16, 32 keys on the A side, the wave's 32 rows on the B side: lane (r, h) = (lane & 31, lane >> 5) holds, for row r,
//            keys 32 t + 8 b + 4 h + e of tile t (b, e = 0..3).
//   P.V:     the 8 k slots of h in MFMA u are the keys that it holds, 16 u + 4 h + (0..3) and 16 u + 8 + 4 h + (0..3): P stays in its lane,
//            the values come out of the row-major tile with the transposing LDS read.
//   Block i + 1 loads during block i, each wave 16 keys of one page.  A wave leaves out the blocks that none of its rows sees.
//   bf16:    direct global->LDS loads.  Chunk c of key row r sits at c ^ k_swizzle(r), of value row r at c ^ v_swizzle(r).
//   8 bits:  codes go through registers, where they become bf16, which holds them exactly, once for the workgroup; a key's scale multiplies its
//            scores, a value's its probability.
//   Bound by the matrix products and by what the chip draws: 2048 tokens over 16384 keys, 32 heads of 128 over 8, 494 to 525 us, 0.98 to 1.04 PFLOP/s with random numbers (by card);
// with zeros, at a higher clock, 398 us, 1296 (the library's product of 8192^3 with random numbers 1307 to 1354).  Of LDS reads it needs as
// much time as of matrix instructions (32 rows a wave).  Tried and slower: scores of block i + 1 ahead of the probabilities of block i (no gain, or spilled),
// 64 rows a wave (868: accumulators move to and fro), eight waves over 256 rows in two phases (537 where this took 521),
// the sum of the probabilities by a matrix instruction with ones (+ 5 %), a copy of the loop without masks (+ 9 %).  32 prompts of up to 512, 16 heads of 64:
// 21.3 us, 69 MB at 3.2 TB/s: 1280 tiles of 1 to 8 blocks, of which 1024 are under way at once; a tile spends 1.3 us in finding itself and 1.7 to 2.9 until its
// first keys are there.
// ---------------------------------------------------------------------------
// (Heads of 64 in 8 bits: three waves a SIMD, with registers for what is converted; 2048 tokens over 16384 keys 439 us, two to four 466, four 684.  Of
// bf16 four: 32 prompts of up to 512 rows 20.7 us, three 22.2, two 25.5.)
template <int D, bool I8>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(I8 && D == 64 ? 3 : 2, I8 && D == 64 ? 3 : 4))) paged_chunks_kernel(PagedArgs g) {
  constexpr int ROWS = 128, KEYS = 64, LEAST = 4;
  constexpr int RB = 2 * D, CH = RB / 16;             // bytes and chunks of a row in LDS
  constexpr int TILE = KEYS * RB;
  constexpr int PER = 1024 / RB, LOADS = 16 / PER;    // rows of a direct load, loads of 16 rows
  constexpr int CB = D, CPER = 1024 / CB, CLOADS = 16 / CPER;  // the same of codes
  constexpr int NT = D / 32;                          // tiles of 32 elements of the output
  // 8 bits: a lane puts chunks 2 c and 2 c + 1 of a row, one after the other; with the two of the row's second half swapped the eight lanes of a row meet in no
  // bank (2048 tokens over 16384 keys 592 -> 580 us).
  constexpr bool SWAPPED = I8 && D == 128;
  constexpr int SCALES = I8 ? 2 * 2 * KEYS * 4 : 0;   // of the keys (times alpha log2 e) and the values of two blocks
  __shared__ __attribute__((aligned(256))) unsigned char lds[4 * TILE + SCALES];  // keys of two blocks, values of two, scales
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, h = lane >> 5;

  __shared__ int unit[kUnitWords];
  if (wave == 0) find_unit<ROWS, KEYS, LEAST>(g, blockIdx.x, unit);
  __syncthreads();
  PagedUnit u;
  if (!take_unit(g, unit, u)) return;
  int low, high, block0, block1;
  unit_keys<ROWS, KEYS>(g, u, low, high, block0, block1);
  const int rows = u.seq.n * g.group, before = u.seq.length - u.seq.n;

  // this lane's row, and the blocks of the workgroup's that its wave's rows see: wave0 .. wave1 - 1
  const int m0 = u.tile * ROWS + wave * 32;
  const int m = m0 + r32, m_ld = m < rows ? m : rows - 1, token = divided(m_ld, g.by_group);
  const int pos = m < rows ? before + token : -1;
  const int first = g.window > 0 ? pos - g.window + 1 : 0;
  const u16* q = g.q + (long long)(u.seq.first + token) * g.q_stride + (u.head * g.group + m_ld - token * g.group) * D;
  bf16x8 qf[D / 16];
#pragma unroll
  for (int dd = 0; dd < D / 16; ++dd) qf[dd] = as_bf16x8(*(const uint4*)(q + dd * 16 + h * 8));
  int wave0 = block1, wave1 = block0, wave_least = -1, wave_high = -1;
  if (m0 < rows) {
    const int last = (m0 + 32 < rows ? m0 + 32 : rows) - 1;
    wave_least = __builtin_amdgcn_readfirstlane(before + divided(m0, g.by_group));
    wave_high = __builtin_amdgcn_readfirstlane(before + divided(last, g.by_group));
    int wave_low = g.window > 0 ? wave_least - g.window + 1 : 0;
    if (wave_low < 0) wave_low = 0;
    wave0 = wave_low / KEYS > block0 ? wave_low / KEYS : block0;
    const int end = wave_high < 0 ? 0 : wave_high / KEYS + 1;
    wave1 = end < block1 ? end : block1;
  }
  wave0 = __builtin_amdgcn_readfirstlane(wave0);
  wave1 = __builtin_amdgcn_readfirstlane(wave1);

  auto k_swizzle = [](int row) { return (row / (256 / RB)) & (CH < 16 ? CH - 1 : 15); };
  auto v_swizzle = [](int row) { return RB == 256 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); };
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_addr_of(lds));
  const int slot_mask = (1 << g.cache.page_shift) - 1;
  const int* table = g.seqs.pages + (long long)u.s * g.seqs.width;
  const int k0 = low & ~15, k1 = high & ~15;
  // of a block this wave loads 16 keys: the first of them, held to what the tile sees, and its page
  auto key_of = [&](int block) {
    const int key = block * KEYS + wave * 16;
    return key < k0 ? k0 : key > k1 ? k1 : key;
  };
  auto page_of = [&](int block) {
    if (high < 0) return 0;
    return table[key_of(block) >> g.cache.page_shift];
  };
  auto row_of = [&](int block, int page) {  // the 16 keys' first row of the cache
    unsigned p = (unsigned)__builtin_amdgcn_readfirstlane(page);
    p = p < g.cache.pages ? p : g.cache.pages - 1;
    return (((long long)p * g.cache.kv_heads + u.head) << g.cache.page_shift) + (key_of(block) & slot_mask);
  };
  // the row that stands in for row r of the 16: of keys outside of what the tile sees the nearest that it does
  auto held = [&](int block, int r) {
    const int key = key_of(block), lo = low - key, hi = high - key;
    return r < lo ? lo : r > hi ? hi : r;
  };
  auto whole = [&](int block) { const int key = block * KEYS + wave * 16; return key >= low && key + 15 <= high; };

  // bf16: to LDS.  The offsets of a lane's pieces of 16 rows that are all there are kept: formed anew they cost the prompt of 2048 rows 13 us of 534.
  const int load_row = lane / CH, load_chunk_ = lane % CH;
  uint32_t load_off[2][LOADS];
#pragma unroll
  for (int n = 0; n < LOADS; ++n) {
    const int r = n * PER + load_row;
    load_off[0][n] = r * RB + (load_chunk_ ^ k_swizzle(r)) * 16;
    load_off[1][n] = r * RB + (load_chunk_ ^ v_swizzle(r)) * 16;
  }
  auto load_tile = [&](auto is_v, int block, long long row) {
    constexpr bool V = decltype(is_v)::value;
    const unsigned char* from = uniform_pointer((V ? g.cache.v : g.cache.k) + row * RB);
    const uint32_t to = ring + (V ? 2 : 0) * TILE + (block & 1) * TILE + wave * (16 * RB);
    if (whole(block)) {
#pragma unroll
      for (int n = 0; n < LOADS; ++n) dma16_so(load_off[V][n], from, to + n * 1024);
      return;
    }
#pragma unroll
    for (int n = 0; n < LOADS; ++n) {
      const int r = n * PER + load_row;
      dma16_so(load_off[V][n] + (uint32_t)((held(block, r) - r) * RB), from, to + n * 1024);
    }
  };
  // 8 bits: to registers, and from there to LDS
  const int code_row = lane / (CB / 16), code_chunk = lane % (CB / 16);
  uint4 codes[2][CLOADS];
  float scale[2];
  auto load_codes = [&](auto is_v, int block, long long row) {
    constexpr bool V = decltype(is_v)::value;
    const unsigned char* from = (V ? g.cache.v : g.cache.k) + row * CB;
#pragma unroll
    for (int n = 0; n < CLOADS; ++n) {
      int r = n * CPER + code_row;
      asm volatile("" : "+v"(r));
      codes[V][n] = *(const uint4*)(from + held(block, r) * CB + code_chunk * 16);
    }
    scale[V] = ((V ? g.cache.v_scale : g.cache.k_scale) + row)[held(block, lane & 15)];
  };
  auto put_codes = [&](auto is_v, int block) {
    constexpr bool V = decltype(is_v)::value;
    unsigned char* to = lds + (V ? 2 : 0) * TILE + (block & 1) * TILE + wave * (16 * RB);
#pragma unroll
    for (int n = 0; n < CLOADS; ++n) {
      int r = n * CPER + code_row;
      asm volatile("" : "+v"(r));
      const int s = V ? v_swizzle(r) : k_swizzle(r);
      const uint4 w = codes[V][n];
      const uint2 a = codes_to_bf16(w.x), b = codes_to_bf16(w.y), c = codes_to_bf16(w.z), d = codes_to_bf16(w.w);
      const int turn = SWAPPED ? code_chunk >> 2 : 0;
      *(uint4*)(to + r * RB + ((2 * code_chunk) ^ s ^ turn) * 16) = make_uint4(a.x, a.y, b.x, b.y);
      *(uint4*)(to + r * RB + ((2 * code_chunk + 1) ^ s ^ turn) * 16) = make_uint4(c.x, c.y, d.x, d.y);
    }
    float* scales = (float*)(lds + 4 * TILE) + (block & 1) * 2 * KEYS + V * KEYS;
    if (lane < 16) scales[wave * 16 + lane] = V ? scale[V] : scale[V] * g.a2;
  };
  using K_TILE = std::false_type;
  using V_TILE = std::true_type;

  f32x16 oacc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) oacc[t][e] = 0.f;
  float ref = kNothing, sum0 = 0.f, sum1 = 0.f;  // ref: bf16 in units of the scores, 8 bits base 2
  const float a2 = I8 ? 1.0f : g.a2;

  const int i16 = lane & 15, dh = (lane >> 4) & 1;
  const int v_row = 4 * h + (i16 >> 2);          // and multiples of 8 further: their swizzle is the same
  uint32_t v_off[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) v_off[t] = v_row * RB + ((4 * t + 2 * dh + ((i16 & 3) >> 1)) ^ v_swizzle(v_row) ^ (SWAPPED ? t >> 1 : 0)) * 16 + (i16 & 1) * 8;
  // chunk 2 dd + h of row 32 t + r: a row's first byte is a multiple of its length, so that the swizzle is one exclusive or
  typedef const __attribute__((address_space(3))) uint4* LdsPtr;
  const uint32_t k_at = ring + r32 * RB + (h ^ k_swizzle(r32)) * 16;
  auto k_part = [&](int slot, int dd, int t) {
    const LdsPtr from = (LdsPtr)(uintptr_t)(((k_at + slot * TILE) ^ (dd * 32 + (SWAPPED ? (dd >> 2) * 16 : 0))) + t * 32 * RB);
    return as_bf16x8(make_uint4(from->x, from->y, from->z, from->w));
  };
  // Which of this lane's keys of a block its row sees: from `least` on `range` + 1, counted from the lane's first (one comparison each).
  struct Seen {
    unsigned least, range;
    __device__ __forceinline__ bool operator()(int key) const { return (unsigned)key - least <= range; }
  };
  auto seen_of = [&](int key0) {
    const int most = pos - key0 - h * 4, least = first - key0 - h * 4;
    Seen seen{most < least ? 0x40000000u : (unsigned)least, most < least ? 0u : (unsigned)(most - least)};
    asm volatile("" : "+v"(seen.least), "+v"(seen.range));  // (else the comparisons of both uses are kept in scalar registers)
    return seen;
  };
  auto block = [&](int i) {
    const int slot = i & 1, key0 = i * KEYS;
    const float* scales = (const float*)(lds + 4 * TILE) + slot * 2 * KEYS;
    f32x16 s[2];
    // Read one step ahead of the matrix instructions, which the barrier keeps the compiler from undoing: 2048 tokens over 16384 keys, heads of 128 in bf16
    // 505 -> 501 us, in 8 bits 609 -> 591; two ahead takes registers that heads of 64 need (21.2 -> 22.5, 32 prompts of up to 512).
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    bf16x8 kf[2][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) kf[0][t] = k_part(slot, 0, t);
#pragma unroll
    for (int dd = 0; dd < D / 16; ++dd) {
      if (dd + 1 < D / 16) {
#pragma unroll
        for (int t = 0; t < 2; ++t) kf[(dd + 1) & 1][t] = k_part(slot, dd + 1, t);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < 2; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[dd & 1][t], qf[dd], dd == 0 ? zero : s[t], 0, 0, 0);
    }
    const bool edge = key0 + KEYS - 1 > wave_least || (g.window > 0 && key0 <= wave_high - g.window);
    if (I8) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const float4 sc = *(const float4*)(scales + t * 32 + b * 8 + h * 4);
          s[t][4 * b] *= sc.x, s[t][4 * b + 1] *= sc.y, s[t][4 * b + 2] *= sc.z, s[t][4 * b + 3] *= sc.w;
        }
    }
    if (edge) {
      const Seen seen = seen_of(key0);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!seen(t * 32 + (e >> 2) * 8 + (e & 3))) s[t][e] = -INFINITY;
    }
    float top = ref;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(fmaxf(top, s[0][e]), s[1][e]);
    {
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(fmaxf(ref, __uint_as_float(sw[0])), __uint_as_float(sw[1]));
    }
    if (__any(top > ref)) {
      const float back = __builtin_amdgcn_exp2f((ref - top) * a2);
      sum0 *= back;
      sum1 *= back;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[t][e] *= back;
      ref = top;
    }
    const float nm2 = ref > kNothing ? -ref * a2 : 0.f;  // (a row that has seen nothing: its scores are minus infinity)
    const uint32_t vs = ring + 2 * TILE + slot * TILE;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      // The values come out of LDS behind the exponentials, for which heads of 64 in bf16 have no registers (505 -> 498 us, with the keys' reads 496; in
      // 8 bits, heads of 64, 434 -> 422).
      constexpr bool AHEAD = D == 128 || I8;
      uint2 values[NT][2];
      auto read_values = [&]() {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint32_t at = vs + v_off[t] + z * 16 * RB;
          values[t][0] = lds_read_tr16(at);
          values[t][1] = lds_read_tr16(at + 8 * RB);
        }
      };
      if (AHEAD) {
        read_values();
        __builtin_amdgcn_sched_barrier(0);
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float sx = s[z >> 1][(z & 1) * 8 + e];
        p[e] = __builtin_amdgcn_exp2f(I8 ? sx + nm2 : fmaf(sx, a2, nm2));
        if (e & 1) sum1 += p[e]; else sum0 += p[e];
      }
      if (I8) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float4 sc = *(const float4*)(scales + KEYS + z * 16 + b * 8 + h * 4);
          p[4 * b] *= sc.x, p[4 * b + 1] *= sc.y, p[4 * b + 2] *= sc.z, p[4 * b + 3] *= sc.w;
        }
        if (edge) {
          const Seen seen = seen_of(key0);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!seen(z * 16 + (e >> 2) * 8 + (e & 3))) p[e] = 0.f;  // (its scale may be NaN)
        }
      }
      // (in bf16, which is as far off as the rounding of the result; in two, as few rows have it, the prompt took 679 us where this takes 510)
      const bf16x8 pf = as_bf16x8(make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])));
      if (!AHEAD) read_values();
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint2 lo = values[t][0], hi = values[t][1];
        oacc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y)), pf, oacc[t], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // Block i is there, and the tiles of the block before are free: block i + 1 into them, its page was looked up during block i - 1.
  const int last = block1 - 1;
  int page_ahead = 0;
  auto load = [&](int i, int page) {
    const long long row = row_of(i, page);
    if (I8) {
      load_codes(K_TILE{}, i, row);
      load_codes(V_TILE{}, i, row);
    } else {
      load_tile(K_TILE{}, i, row);
      load_tile(V_TILE{}, i, row);
    }
  };
  if (block0 < block1) {
    page_ahead = page_of(block0 < last ? block0 + 1 : last);
    load(block0, page_of(block0));
    for (int i = block0; i < block1; ++i) {
      if (I8) {
        put_codes(K_TILE{}, i);
        put_codes(V_TILE{}, i);
      }
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __syncthreads();
      if (i < last) {
        load(i + 1, page_ahead);
        if (i + 1 < last) page_ahead = page_of(i + 2);
      }
      if (i >= wave0 && i < wave1) block(i);
    }
  }
  put_unit_item(g, u);
  if (m0 >= rows) return;
  if (!I8) {
    bool odd = false;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) odd |= not_finite(oacc[t][e]);
    if (__any(odd)) {
      for (int r = 0; r < 32; ++r)
        if (m0 + r < rows) careful_row<ROWS, D>(g, u, m0 + r, block0 * KEYS, block1 * KEYS);
      return;
    }
  }
  float sum = sum0 + sum1;
  sum += __shfl_xor(sum, 32, 64);
  if (m >= rows) return;
  if (u.slot >= 0) {
    const long long to = (long long)u.slot * ROWS + wave * 32 + r32;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *(float4*)(g.part + to * D + t * 32 + b * 8 + h * 4) = make_float4(oacc[t][4 * b], oacc[t][4 * b + 1], oacc[t][4 * b + 2], oacc[t][4 * b + 3]);
    if (h == 0) g.stat[to] = make_float2(ref > kNothing ? ref * a2 : kNothing, sum);
    return;
  }
  const float inv = pos < 0 ? 0.f : 1.0f / sum;
  u16* o = g.o + ((long long)(u.seq.first + token) * g.heads + u.head * g.group + m - token * g.group) * D;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int b = 0; b < 4; b += 2) {  // (the two lanes of a row exchange, for whole 16 bytes a lane: 32 prompts of up to 512 rows 22.0 -> 21.5 us)
      uint32_t w[2][2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) w[x][y] = pack_bf16x2(oacc[t][4 * (b + x) + 2 * y] * inv, oacc[t][4 * (b + x) + 2 * y + 1] * inv);
      const auto s0 = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
      *(uint4*)(o + t * 32 + (b + h) * 8) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
    }
}

}  // namespace nimble
#endif
