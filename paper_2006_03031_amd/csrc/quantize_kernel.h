// Rows to 8-bit codes and one scale each.
#ifndef NIMBLE_QUANTIZE_KERNEL_H_
#define NIMBLE_QUANTIZE_KERNEL_H_
#include "device_common.h"

namespace nimble {

// ---------------------------------------------------------------------------
// scale = a / 127, q = 127 x / a to the nearest integer (ties to even) with a = max |x| of the row: the exactly rounded code, so that
// it does not depend on how the quotient is computed.  t = x (127 / a) in f32 is off by less than 2^-15 (|t| <= 127, two
// roundings of 2^-24 and one of the reciprocal).  Where a t is that close to the border of two codes (bf16: x = a / 2 is one)
// the remainder e = 127 x - r a decides, r the code next to t: a step further if 2 |e| > a, or = a with r odd.  For bf16
// it is exact in f32 (127 x and r a have 15 bits each, and a code r != 0 keeps their exponents within 8 of each other; for
// r = 0 it is 127 x); for f32 it is taken in f64, whose products of 24 + 8 bits are exact.
//   Rows below 2^-100 are taken times 2^100 first, since 127 / a would overflow, and rows beyond 2^100 times 2^-100, since 127 x would
// (exact but for elements so small that their code is 0 anyway); rows with an infinity or a NaN get codes 0
//   and scale NaN, which makes every result of the row NaN.
//   Bound: memory (2 or 4 bytes read and one written per element): 8177 x 4096 bf16 21.6 us, 4.7 TB/s of the 5.2 that a copy reaches (75 us with
// the border decided in f64 for every element group and values held as f32); 8177 x 1024 9.8-11.7, 8177 x 8192 38.8, 4096 x 16384 52 (3.8 TB/s; with
// eight groups held two waves per SIMD are left), 4096 x 4096 f32 15.8, 4096 x 16384 f32 74.  A row stays in registers, as it was read, between the
// maximum and the codes; of one longer than 16384 the rest is read twice: 2000 x 30522 bf16 74 us, 2.5 TB/s.
// ---------------------------------------------------------------------------
struct QuantizeArgs {
  const void* x;
  signed char* q;
  float* scale;
  long long rows;
  int K, cols;
};

// Eight elements of a row as they are in memory.
template <bool F32>
struct Raw8 {
  uint4 part[F32 ? 2 : 1];
  __device__ __forceinline__ float value(int i) const {
    const uint4& p = part[F32 ? i >> 2 : 0];
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
    if (F32) return __uint_as_float(w[i & 3]);
    return __uint_as_float((i & 1) ? w[(i >> 1) & 3] & 0xffff0000u : w[(i >> 1) & 3] << 16);
  }
};
// Elements at .. at + 7 of a row of K, those past its end zero.  Any alignment.
template <bool F32>
__device__ __forceinline__ Raw8<F32> load_raw8(const void* row, int at, int K) {
  Raw8<F32> v;
  const int n = K - at;
  if (n >= 8) {
    __builtin_memcpy(&v, F32 ? (const void*)((const float*)row + at) : (const void*)((const u16*)row + at), sizeof v);
  } else {
    uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i) {
      if (i >= n) continue;
      if (F32)
        w[i] = ((const uint32_t*)row)[at + i];
      else
        w[i >> 1] |= (uint32_t)((const u16*)row)[at + i] << (16 * (i & 1));
    }
    v.part[0] = make_uint4(w[0], w[1], w[2], w[3]);
    if (F32) v.part[F32 ? 1 : 0] = make_uint4(w[4], w[5], w[6], w[7]);
  }
  return v;
}

// WAVES waves per row, each thread holds NV groups of 8 consecutive elements; what a row has beyond is read twice.
template <bool F32, int WAVES, int NV>
__global__ void __launch_bounds__(256) quantize_rows_kernel(QuantizeArgs g) {
  constexpr int TPR = WAVES * 64, ROWS = 256 / TPR;
  constexpr float kRound = 12582912.0f;  // 1.5 2^23: a sum with it is rounded to the integer that its low byte is
  __shared__ uint32_t tops[4];
  const int tid = threadIdx.x % TPR;
  const bool whole = (g.cols & 7) == 0;
  for (long long row = (long long)blockIdx.x * ROWS + threadIdx.x / TPR; row < g.rows; row += (long long)gridDim.x * ROWS) {
    const void* x = F32 ? (const void*)((const float*)g.x + row * g.K) : (const void*)((const u16*)g.x + row * g.K);
    uint32_t top = 0;  // of the bits of |x|: these order as the values do, infinities and NaN last
    auto look = [&](const Raw8<F32>& v) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v.value(i)) & 0x7fffffffu);
    };
    Raw8<F32> held[NV];
#pragma unroll
    for (int c = 0; c < NV; ++c) held[c] = load_raw8<F32>(x, (c * TPR + tid) * 8, g.K);
    for (int at = (NV * TPR + tid) * 8; at < g.K; at += TPR * 8) look(load_raw8<F32>(x, at, g.K));
#pragma unroll
    for (int c = 0; c < NV; ++c) look(held[c]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if (WAVES > 1) {
      __syncthreads();  // (the row before has been read)
      if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
      __syncthreads();
      top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    }
    const bool finite = top < 0x7f800000u;
    const float a0 = __uint_as_float(top);
    const float lift = a0 < 7.8886091e-31f ? 1.2676506e30f : a0 > 1.2676506e30f ? 7.8886091e-31f : 1.0f;  // 2^-100, 2^100
    const float a = finite && top ? a0 * lift : 1.0f;
    const float inv = finite && top ? 127.0f / a : 0.0f;
    if (tid == 0) g.scale[row] = finite ? a0 / 127.0f : __uint_as_float(0x7fc00000u);
    signed char* q = g.q + row * g.cols;
    auto put = [&](int at, const Raw8<F32>& v) {
      uint32_t m[8];
      float far = 0.0f;  // the furthest that a t is from its code
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float t = v.value(i) * lift * inv, sum = t + kRound;
        m[i] = __float_as_uint(sum);
        far = fmaxf(far, fabsf(t - (sum - kRound)));
      }
      if (far > 0.49993896f) {  // 1/2 - 2^-14
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float r = __uint_as_float(m[i]) - kRound;
          const float s = v.value(i) * lift;
          float sign;
          bool over, even;
          if (F32) {
            const double e = 127.0 * (double)s - (double)r * (double)a, h = 0.5 * (double)a;
            over = fabs(e) > h, even = fabs(e) == h, sign = e < 0 ? -1.0f : 1.0f;
          } else {
            const float e = fmaf(-r, a, 127.0f * s), h = 0.5f * a;
            over = fabsf(e) > h, even = fabsf(e) == h, sign = e < 0 ? -1.0f : 1.0f;
          }
          if (over || (even && ((int)r & 1))) r += sign;
          m[i] = __float_as_uint(r + kRound);
        }
      }
      uint32_t code[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(m[4 * h + 1], m[4 * h], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(m[4 * h + 3], m[4 * h + 2], 0x04000c0cu);
        code[h] = finite ? lo | hi : 0u;
      }
      if (whole) {
        *(uint2*)(q + at) = make_uint2(code[0], code[1]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (at + i < g.cols) q[at + i] = (signed char)(code[i >> 2] >> (8 * (i & 3)));
      }
    };
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const int at = (c * TPR + tid) * 8;
      if (at < g.cols) put(at, held[c]);
    }
    for (int at = (NV * TPR + tid) * 8; at < g.cols; at += TPR * 8) put(at, load_raw8<F32>(x, at, g.K));
  }
}

}  // namespace nimble
#endif
