// Rows to 8-bit codes and one scale each.
#ifndef NIMBLE_QUANTIZE_KERNEL_H_
#define NIMBLE_QUANTIZE_KERNEL_H_
#include "device_common.h"

namespace nimble {

// ---------------------------------------------------------------------------
// scale = a / 127, q = 127 x / a to the nearest integer (ties to even) with a = max |x| of the row: the exactly rounded code, so that
// it does not depend on how the quotient is computed.  t = x (127 / a) in f32 is off by less than 2^-15 (|t| <= 127, two
// roundings of 2^-24 and one of the reciprocal); a t that close to the border of two codes is decided by the sign of
// 127 x - (border) a, whose two products are exact in f64 (24 + 8 bits).
//   Rows below 2^-100 are taken times 2^100 first (exact), since 127 / a would overflow; rows with an infinity or a NaN get codes 0
//   and scale NaN, which makes every result of the row NaN.
//   Bound: memory (2 or 4 bytes read and one written per element).  A row stays in registers between the two passes over it.
// ---------------------------------------------------------------------------
struct QuantizeArgs {
  const void* x;
  signed char* q;
  float* scale;
  long long rows;
  int K, cols;
};

__device__ __forceinline__ float quantize_code(float x, float inv, float a) {
  const float t = x * inv;
  float r = rintf(t);
  if (fabsf(fabsf(t - r) - 0.5f) < 6.1035156e-5f) {  // 2^-14
    const float half = t < r ? r - 0.5f : r + 0.5f;
    const double d = 127.0 * (double)x - (double)half * (double)a;
    const float down = half - 0.5f, up = half + 0.5f;
    r = d > 0 ? up : d < 0 ? down : (((int)down & 1) ? up : down);
  }
  return r;
}

template <bool F32>
__device__ __forceinline__ void load_values(const void* row, int at, int K, float (&v)[8]) {
  if (at + 8 <= K) {
    if (F32) {
      const float* p = (const float*)row + at;
      __builtin_memcpy(v, p, 32);
    } else {
      const uint4 u = load8_unaligned((const u16*)row + at);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = at + i < K ? (F32 ? ((const float*)row)[at + i] : bf2f(((const u16*)row)[at + i])) : 0.0f;
  }
}

// WAVES waves per row, each thread holds NV groups of 8 consecutive elements; longer rows are read twice.
template <bool F32, int WAVES, int NV>
__global__ void __launch_bounds__(256) quantize_rows_kernel(QuantizeArgs g) {
  constexpr int TPR = WAVES * 64, ROWS = 256 / TPR;
  __shared__ uint32_t tops[4];
  const int tid = threadIdx.x % TPR;
  for (long long row = (long long)blockIdx.x * ROWS + threadIdx.x / TPR; row < g.rows; row += (long long)gridDim.x * ROWS) {
    const void* x = F32 ? (const void*)((const float*)g.x + row * g.K) : (const void*)((const u16*)g.x + row * g.K);
    float v[NV][8];
    uint32_t top = 0;  // of the bits of |x|: these order as the values do, infinities and NaN last
    for (int at = (NV * TPR + tid) * 8; at < g.K; at += TPR * 8) {
      float far[8];
      load_values<F32>(x, at, g.K, far);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(far[i]) & 0x7fffffffu);
    }
#pragma unroll
    for (int c = 0; c < NV; ++c) load_values<F32>(x, (c * TPR + tid) * 8, g.K, v[c]);
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[c][i]) & 0x7fffffffu);
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
    const float lift = a0 < 7.8886091e-31f ? 1.2676506e30f : 1.0f;  // 2^-100, 2^100
    const float a = finite && top ? a0 * lift : 1.0f;
    const float inv = finite && top ? 127.0f / a : 0.0f;
    if (tid == 0) g.scale[row] = finite ? a0 / 127.0f : __uint_as_float(0x7fc00000u);
    signed char* q = g.q + row * g.cols;
    const bool whole = (g.cols & 7) == 0;
    auto put = [&](int at, const float (&w)[8]) {
      uint32_t code[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float c = finite ? quantize_code(w[i] * lift, inv, a) : 0.0f;
        code[i >> 2] |= ((uint32_t)(int)c & 0xffu) << (8 * (i & 3));
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
      if (at < g.cols) put(at, v[c]);
    }
    for (int at = (NV * TPR + tid) * 8; at < g.cols; at += TPR * 8) {
      float far[8];
      load_values<F32>(x, at, g.K, far);
      put(at, far);
    }
  }
}

}  // namespace nimble
#endif
