// What the paged cache's operators share between host and device: arguments, limits.
#ifndef NIMBLE_CACHE_INTERNAL_H_
#define NIMBLE_CACHE_INTERNAL_H_
#include <array>
#include <initializer_list>

#include "nimble_internal.h"

namespace nimble {

// nimble_sequences and nimble_cache as the kernels take them.
struct SequencesArgs {
  const long long* offsets;
  const long long* lengths;
  const int* pages;
  int count, width, rows;
};
// x / d for x < 2^30 and d <= 2^16 as (2 x magic / 2^32) >> shift: shift = floor(log2 d), magic = ceil(2^(31 + shift) / d), whose excess e = magic d - 2^(31 + shift)
// is at most d - 1 < 2^(shift + 1), so that x e < 2^(31 + shift), which is less than what a quotient can be off by.
struct Divisor {
  unsigned magic, shift;
};
inline Divisor divisor_of(int64_t d) {
  unsigned shift = 0;
  while ((d >> shift) > 1) ++shift;
  return Divisor{(unsigned)(((1ull << (31 + shift)) + (uint64_t)d - 1) / (uint64_t)d), shift};
}

struct CacheArgs {
  unsigned char* k;
  unsigned char* v;
  float* k_scale;
  float* v_scale;
  unsigned pages;
  int kv_heads, page_shift;
};

// A launch is of fewer than 2^32 threads.
constexpr int64_t kMostPagedGrid = 1 << 23;
// Sequences are looked for 64 by 64 (SpanWalk, find_unit), positions and rows are 32-bit numbers.
constexpr int64_t kMostSequences = 1 << 16, kMostPositions = 1ll << 30, kMostRows = 1ll << 24;
constexpr int kPagedItemWords = 12;
constexpr int kPagedBlockKeys = 32;  // of the kernel of few rows

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// `rows` rows of `bytes` bytes, `stride` bytes apart; nothing where `at` is null.
struct Extent {
  const char* name;
  const void* at;
  int64_t rows, bytes, stride;
};
inline Extent extent(const char* name, const void* at, int64_t bytes) { return Extent{name, at, 1, bytes, bytes}; }
// Rows of bf16, in elements.  (Beyond 2^40 of them apart the second lies behind all memory as well.)
inline Extent extent(const char* name, const void* at, int64_t rows, int64_t row, int64_t stride) {
  return rows == 1 || stride == row ? extent(name, at, rows * row * 2) : Extent{name, at, rows, row * 2, (stride < 1ll << 40 ? stride : 1ll << 40) * 2};
}
// Outputs that share memory with an operand or with each other are refused.
int check_apart(const char* what, std::initializer_list<Extent> outputs, std::initializer_list<Extent> operands);
std::array<Extent, 4> cache_extents(const nimble_cache& c);
std::array<Extent, 3> sequences_extents(const nimble_sequences& s);

int check_hip_launch(const char* what);

int check_cache(const nimble_cache* c);
int check_sequences(const nimble_sequences* s, int64_t page);
CacheArgs cache_args(const nimble_cache& c);
SequencesArgs sequences_args(const nimble_sequences& s);

}  // namespace nimble
#endif
