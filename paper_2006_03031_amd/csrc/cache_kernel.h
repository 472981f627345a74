// Rotary positions, and rows into and out of a paged cache.
#ifndef NIMBLE_CACHE_KERNEL_H_
#define NIMBLE_CACHE_KERNEL_H_
#include "cache_device.h"

namespace nimble {

struct RotaryArgs {
  const uint16_t* x;
  const long long* positions;
  const float2* table;
  uint16_t* y;
  long long x_stride, y_stride, table_rows, T;
  int H, D, R;
};

struct CacheWriteArgs {
  CacheArgs cache;
  SequencesArgs seqs;
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* q;   // or nullptr
  uint16_t* q_out;
  const float2* table; // or nullptr
  long long k_stride, v_stride, q_stride, table_rows;
  int heads, R, rows_each;
};

struct CacheReadArgs {
  CacheArgs cache;
  SequencesArgs seqs;
  void* k_out;
  void* v_out;
  int rows_each;
};

// ---------------------------------------------------------------------------
// The table of angles: made once, in f64 throughout.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(256)
    rotary_table_kernel(float2* table, long long count, int R, double base, double factor, double trained, double low, double high, double magnitude) {
  for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < count; at += (long long)gridDim.x * 256) {
    const long long p = at / R;
    const int i = (int)(at - p * R);
    double f = pow(base, -(double)i / (double)R);
    const double turns = trained * f * 0.15915494309189535;  // 1 / 2 pi
    double keep = (turns - low) / (high - low);
    keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
    if (trained == 0) keep = 0;
    f *= keep + (1 - keep) / factor;
    double s, c;
    sincos((double)p * f, &s, &c);
    table[at] = make_float2((float)(magnitude * c), (float)(magnitude * s));
  }
}

// ---------------------------------------------------------------------------
// y_a = x_a c - x_b s, y_b = x_b c + x_a s.  A thread holds 8 pairs as they lie in memory: two chunks of 8 elements half the turned part
// apart, or two neighbouring ones where pairs are neighbours.  In f32, rounded once to bf16: one product is
// rounded to 24 bits and the sum with the other, so that ahead of bf16 a result is off by 2^-23 (|x_a c| + |x_b s|) at most, which can be more than a
// step of it where the two cancel.
//   Bound by memory: 8177 rows of 32 heads of 128 in 26.2 us, 136 MB at 5.2 TB/s, what a copy of 1 GiB reaches; one row of 16 heads 1.6, a launch and two
// loads one behind the other.  (Loads or stores past the caches were slower.)
// ---------------------------------------------------------------------------
struct Chunk {  // 8 bf16
  uint32_t w[4];
  __device__ __forceinline__ float value(int i) const { return of_pair(w[i >> 1], i & 1); }
};
__device__ __forceinline__ Chunk load_chunk(const u16* p) {
  const uint4 v = *(const uint4*)p;
  return Chunk{{v.x, v.y, v.z, v.w}};
}
__device__ __forceinline__ void store_chunk(u16* p, const Chunk& c) { *(uint4*)p = make_uint4(c.w[0], c.w[1], c.w[2], c.w[3]); }

// The 16 values of two chunks turned by eight rows of the table (those of pairs first, first + 1, ...).
template <bool INTERLEAVED, typename F>
__device__ __forceinline__ void turn(const Chunk& a, const Chunk& b, const float4* table, F (&ya)[8], F (&yb)[8]) {
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const float4 t = table[h];  // two pairs
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = 2 * h + e;
      const F c = e ? t.z : t.x, s = e ? t.w : t.y;
      if (INTERLEAVED) {
        const Chunk& x = i < 4 ? a : b;
        const F u = x.value(2 * (i & 3)), v = x.value(2 * (i & 3) + 1);
        (i < 4 ? ya : yb)[2 * (i & 3)] = fma(u, c, -(v * s));
        (i < 4 ? ya : yb)[2 * (i & 3) + 1] = fma(v, c, u * s);
      } else {
        const F u = a.value(i), v = b.value(i);
        ya[i] = fma(u, c, -(v * s));
        yb[i] = fma(v, c, u * s);
      }
    }
  }
}
template <typename F>
__device__ __forceinline__ Chunk rounded(const F (&y)[8]) {
  Chunk c;
#pragma unroll
  for (int i = 0; i < 4; ++i) c.w[i] = pack_bf16x2((float)y[2 * i], (float)y[2 * i + 1]);
  return c;
}

// Which two chunks of a head of `chunks` a lane holds: turned ones `half` chunks apart (neighbours where INTERLEAVED), then the rest.
template <bool INTERLEAVED>
__device__ __forceinline__ void chunks_of(int l, int half, int& a, int& b) {
  a = INTERLEAVED || l >= half ? 2 * l : l;
  b = INTERLEAVED || l >= half ? 2 * l + 1 : l + half;
}

// Rows of any width and alignment: a thread an element pair or a copied element.
template <bool INTERLEAVED>
__global__ void __launch_bounds__(256) rotary_any_kernel(RotaryArgs g) {
  const int per = g.R + (g.D - 2 * g.R);
  const long long count = g.T * g.H * per;
  for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < count; at += (long long)gridDim.x * 256) {
    const long long head = at / per, t = head / g.H;
    const int i = (int)(at - head * per), h = (int)(head - t * g.H);
    const u16* x = g.x + t * g.x_stride + (long long)h * g.D;
    u16* y = g.y + t * g.y_stride + (long long)h * g.D;
    if (i >= g.R) {
      y[g.R + i] = x[g.R + i];
      continue;
    }
    long long p = g.positions[t];
    p = p < 0 ? 0 : p >= g.table_rows ? g.table_rows - 1 : p;
    const float2 cs = g.table[p * g.R + i];
    const int a = INTERLEAVED ? 2 * i : i, b = INTERLEAVED ? 2 * i + 1 : i + g.R;
    const float u = bf2f(x[a]), v = bf2f(x[b]);
    y[a] = f2bf(fmaf(u, cs.x, -(v * cs.y)));
    y[b] = f2bf(fmaf(v, cs.x, u * cs.y));
  }
}

// Rows of whole chunks.  A thread two chunks of one head: `per` threads a head (D / 16).
template <bool INTERLEAVED>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryArgs g) {
  const int per = g.D >> 4, half = INTERLEAVED ? 0 : g.R >> 3;
  const long long count = g.T * g.H * per;
  for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < count; at += (long long)gridDim.x * 256) {
    const long long head = at / per, t = head / g.H;
    const int l = (int)(at - head * per), h = (int)(head - t * g.H);
    int a, b;
    chunks_of<INTERLEAVED>(l, half, a, b);
    const u16* x = g.x + t * g.x_stride + (long long)h * g.D;
    u16* y = g.y + t * g.y_stride + (long long)h * g.D;
    Chunk ca = load_chunk(x + a * 8), cb = load_chunk(x + b * 8);
    const int first = l * 8;  // of this lane's pairs
    if (first < g.R) {
      long long p = g.positions[t];
      p = p < 0 ? 0 : p >= g.table_rows ? g.table_rows - 1 : p;
      float ya[8], yb[8];
      turn<INTERLEAVED>(ca, cb, (const float4*)(g.table + p * g.R + first), ya, yb);
      ca = rounded(ya);
      cb = rounded(yb);
    }
    store_chunk(y + a * 8, ca);
    store_chunk(y + b * 8, cb);
  }
}

// ---------------------------------------------------------------------------
// The places of up to 16 neighbouring rows of a batch, worked out by one wave for its workgroup: a chain of three loads (offsets; lengths; pages)
// that every row would walk by itself otherwise.  36860 rows of 8 heads of 128 in 8 bits read back: a row a workgroup 57.7 us, 16 rows, side by side
// in a wave, 43.5.  Written, 8448 rows of 16 heads of 64 of each take 23 to 25 us either way.
// ---------------------------------------------------------------------------
constexpr int kMostPlaces = 16;
struct Places {
  long long row[kMostPlaces];   // of the cache, for head 0; -1: none, -2: a row of no sequence
  int position[kMostPlaces];
};
__device__ __forceinline__ void find_places(const CacheArgs& c, const SequencesArgs& g, int t0, int n, Places& places) {
  const int lane = threadIdx.x & 63;
  int s = -1;
  if (g.count <= 64) {
    const long long end = lane < g.count ? g.offsets[lane + 1] : 0x7fffffffffffffffll, begin = g.offsets[0];
    for (int r = 0; r < n; ++r) {
      const int passed = __popcll(__ballot(end <= t0 + r));
      if (lane == r) s = passed < g.count && (passed > 0 || begin <= t0 + r) ? passed : -1;
    }
  } else {
    for (int r = 0; r < n; ++r) {
      const int found = sequence_at(g, t0 + r);
      if (lane == r) s = found;
    }
  }
  if (lane >= n) return;
  long long row = -2;
  int p = 0;
  if (s >= 0) {
    const Sequence q = sequence_of(g, s, c.page_shift);
    p = q.length - q.n + (t0 + lane - q.first);
    row = cache_row(c, g, s, p);
  }
  places.row[lane] = row;
  places.position[lane] = p;
}

// ---------------------------------------------------------------------------
// New rows into the cache.  A workgroup takes `rows_each` neighbouring rows of the batch; D / 16 lanes a head, of queries, keys and values alike, each
// with two chunks as above.  8 bits: scale = a / 127, code = 127 x / a to the nearest integer, ties to even, with a = max |x| of the head, all of it in
// f64, where a turned key is exact to 2^-50 or so: the code does not depend on how the quotient is computed, since one within 1e-12 of
// the border of two is decided by the quotient itself.  Heads with an infinity or a NaN, or a scale beyond f32: codes 0, scale NaN.
//   Bound by memory where there are many rows: 8448 of 16 + 16 + 16 heads of 64 in bf16 24.4 us, 104 MB at 4.3 TB/s.  61 rows of 32 + 8 + 8 heads of 128 in
// 8 bits 4.1 us (replayed in a graph), four loads one behind the other (offsets, lengths, pages, table) and the f64 arithmetic of a head.
// ---------------------------------------------------------------------------
__device__ __forceinline__ int code_of(double x, double a, double inv) {
  const double t = x * inv;
  double r = rint(t);
  if (fabs(fabs(t - r) - 0.5) < 1e-12) r = rint(127.0 * x / a);
  return (int)r;
}

template <int D, bool I8, bool INTERLEAVED>
__global__ void __launch_bounds__(256) cache_write_kernel(CacheWriteArgs g) {
  constexpr int LANES = D / 16;
  __shared__ Places places;
  const int t0 = blockIdx.x * g.rows_each, n = g.seqs.rows - t0 < g.rows_each ? g.seqs.rows - t0 : g.rows_each;
  const int G = g.cache.kv_heads, queries = g.q ? g.heads : 0, heads = queries + 2 * G;
  const int l = threadIdx.x % LANES;
  int a, b;
  chunks_of<INTERLEAVED>(l, INTERLEAVED ? 0 : g.R >> 3, a, b);
  const bool turned = g.table && l * 8 < g.R;
  // Heads of all rows one after the other: this lane's, and the next 256 / LANES further (times the workgroups that share the rows).  A head is loaded ahead of its turn, the first ahead of
  // the places.
  constexpr int STEP = 256 / LANES;
  const int step = STEP * gridDim.y, step_r = step / heads, step_h = step - step_r * heads;
  int next_h = blockIdx.y * STEP + threadIdx.x / LANES, next_r = next_h / heads;
  next_h -= next_r * heads;
  Chunk next_a{}, next_b{};
  auto load = [&]() {
    if (next_r >= n) return;
    const int t = t0 + next_r, h = next_h;
    const u16* x = (h < queries ? g.q + t * g.q_stride + h * D : h < queries + G ? g.k + t * g.k_stride + (h - queries) * D
                                                                                  : g.v + t * g.v_stride + (h - queries - G) * D);
    next_a = load_chunk(x + a * 8);
    next_b = load_chunk(x + b * 8);
  };
  load();
  if (threadIdx.x < 64) find_places(g.cache, g.seqs, t0, n, places);
  __syncthreads();
  while (next_r < n) {
    const int r = next_r, h = next_h;
    Chunk ca = next_a, cb = next_b;
    next_r += step_r;
    next_h += step_h;
    if (next_h >= heads) next_h -= heads, ++next_r;
    load();
    const long long row = places.row[r];
    if (row == -2) continue;
    const int t = t0 + r;
    const int kind = h < queries ? 0 : h < queries + G ? 1 : 2;  // query, key, value
    const int head = kind == 0 ? h : h - queries - (kind == 2 ? G : 0);
    if (kind != 0 && row < 0) continue;
    long long at = places.position[r];
    at = at < 0 ? 0 : at >= g.table_rows ? g.table_rows - 1 : at;
    const float4* table = (const float4*)(g.table + at * g.R + l * 8);
    if (kind == 0 || !I8) {
      if (kind != 2 && turned) {
        float ya[8], yb[8];
        turn<INTERLEAVED>(ca, cb, table, ya, yb);
        ca = rounded(ya);
        cb = rounded(yb);
      }
      u16* y = kind == 0 ? g.q_out + ((long long)t * g.heads + head) * D
                         : (u16*)(kind == 1 ? g.cache.k : g.cache.v) + (row + ((long long)head << g.cache.page_shift)) * D;
      store_chunk(y + a * 8, ca);
      store_chunk(y + b * 8, cb);
      continue;
    }
    double ya[8], yb[8];
    if (kind == 1 && turned) {
      turn<INTERLEAVED>(ca, cb, table, ya, yb);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) ya[i] = ca.value(i), yb[i] = cb.value(i);
    }
    double top = 0;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      top = fmax(top, fmax(fabs(ya[i]), fabs(yb[i])));
      odd |= !(fabs(ya[i]) < INFINITY) || !(fabs(yb[i]) < INFINITY);
    }
    if (odd) top = INFINITY;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) top = fmax(top, __shfl_xor(top, o, 64));  // (the lanes of a head take the same branches)
    // (a turned key may pass f32 where its scale does not: the quotient in f64 then; a scale that passes it too is no scale)
    const float scale = top > (double)3.40282347e38f ? (float)(top / 127.0) : (float)top / 127.0f;
    const bool finite = scale < INFINITY;
    const double inv = finite && top > 0 ? 127.0 / top : 0.0;
    uint32_t code[4] = {0, 0, 0, 0};
    if (inv > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        code[i >> 2] |= (uint32_t)(code_of(ya[i], top, inv) & 255) << (8 * (i & 3));
        code[2 + (i >> 2)] |= (uint32_t)(code_of(yb[i], top, inv) & 255) << (8 * (i & 3));
      }
    }
    const long long to = row + ((long long)head << g.cache.page_shift);
    unsigned char* y = (kind == 1 ? g.cache.k : g.cache.v) + to * D;
    *(uint2*)(y + a * 8) = make_uint2(code[0], code[1]);
    *(uint2*)(y + b * 8) = make_uint2(code[2], code[3]);
    if (l == 0) (kind == 1 ? g.cache.k_scale : g.cache.v_scale)[to] = finite ? scale : __uint_as_float(0x7fc00000u);
  }
}

// ---------------------------------------------------------------------------
// Rows back out of the cache: 8 elements a thread, `rows_each` neighbouring rows a workgroup.  As many rows of one head as a wave holds lie side by side
// in it: they are neighbours in the cache, where they are read (past the caches, once), and whole lines in the output.
//   Bound by memory: 36860 rows of 8 heads of 128 in 8 bits 43.5 us, 229 MB at 5.3 TB/s; 999 of 12 heads of 64 in bf16 3.8 us.
// ---------------------------------------------------------------------------
template <int D, bool I8, bool F32>
__global__ void __launch_bounds__(256) cache_read_kernel(CacheReadArgs g) {
  constexpr int LANES = D / 8, MOST = 64 / LANES;
  __shared__ Places places;
  const int t0 = blockIdx.x * g.rows_each, n = g.seqs.rows - t0 < g.rows_each ? g.seqs.rows - t0 : g.rows_each;
  if (threadIdx.x < 64) find_places(g.cache, g.seqs, t0, n, places);
  __syncthreads();
  const int G = g.cache.kv_heads;
  const int beside = g.rows_each >= MOST ? MOST : 1;                    // rows of a wave; its other lanes have other heads
  const int c = threadIdx.x % LANES, x = threadIdx.x / LANES, r0 = x % beside, h0 = x / beside, step = 256 / LANES / beside;
  for (int h = h0 + blockIdx.y * step; h < 2 * G; h += step * gridDim.y) {
    const int head = h < G ? h : h - G;
    const unsigned char* from = h < G ? g.cache.k : g.cache.v;
    const float* scales = h < G ? g.cache.k_scale : g.cache.v_scale;
    void* out = h < G ? g.k_out : g.v_out;
#pragma unroll 4
    for (int r = r0; r < n; r += beside) {
      if (places.row[r] < 0) continue;
      const long long row = places.row[r] + ((long long)head << g.cache.page_shift);
      const unsigned char* at = from + (row * D + c * 8) * (I8 ? 1 : 2);
      const long long to = ((long long)(t0 + r) * G + head) * D + c * 8;
      typedef unsigned Words __attribute__((ext_vector_type(I8 ? 2 : 4)));
      const Words w = __builtin_nontemporal_load((const Words*)at);
      float y[8];
      if constexpr (I8) {
        const float scale = scales[row];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (float)(signed char)(w[i >> 2] >> (8 * (i & 3))) * scale;
      } else {
        const Chunk ch{{w[0], w[1], w[2], w[3]}};
        if (!F32) {
          store_chunk((u16*)out + to, ch);
          continue;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = ch.value(i);
      }
      if (F32) {
        *(float4*)((float*)out + to) = make_float4(y[0], y[1], y[2], y[3]);
        *(float4*)((float*)out + to + 4) = make_float4(y[4], y[5], y[6], y[7]);
      } else {
        store_chunk((u16*)out + to, rounded(y));
      }
    }
  }
}

}  // namespace nimble
#endif
