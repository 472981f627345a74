// Where the rows of a batch and their keys and values are.
#ifndef NIMBLE_CACHE_DEVICE_H_
#define NIMBLE_CACHE_DEVICE_H_

#include "cache_internal.h"
#include "device_common.h"

namespace nimble {

// ---------------------------------------------------------------------------
// Where a row of a batch belongs.  Nothing that the device holds leads outside the tensors: offsets, lengths and pages are held to
// their ranges wherever they are used.
// ---------------------------------------------------------------------------
struct Sequence {
  int first, n, length;  // its rows, and its tokens with them
};
__device__ __forceinline__ Sequence sequence_of(const SequencesArgs& g, int s, int page_shift) {
  const long long lo = g.offsets[s], hi = g.offsets[s + 1], len = g.lengths[s], most = (long long)g.width << page_shift;
  Sequence q;
  q.first = (int)(lo < 0 ? 0 : lo > g.rows ? g.rows : lo);
  const int last = (int)(hi < q.first ? q.first : hi > g.rows ? g.rows : hi);
  q.n = last - q.first;
  q.length = (int)(len < 0 ? 0 : len > most ? most : len);
  return q;
}

// The sequence of row t (of those that have rows), or -1; the same in all lanes.  offsets[s + 1] <= t of as many s as there are ahead of
// it: 64 of them a step, after a step over every 64th (and 4096th) where there are more.
__device__ __forceinline__ int sequence_at(const SequencesArgs& g, int t) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int span = g.count > 4096 ? 4096 : g.count > 64 ? 64 : 1;; span >>= 6) {
    const long long s = base + (long long)(lane + 1) * span - 1;    // the last of this lane's span
    const bool passed = s < g.count && g.offsets[s + 1] <= t;
    base += __popcll(__ballot(passed)) * span;
    if (span == 1) break;
  }
  return base < g.count && g.offsets[base] <= t ? base : -1;
}

// One of two neighbouring bf16.
__device__ __forceinline__ float of_pair(uint32_t w, int i) { return __uint_as_float(i ? w & 0xffff0000u : w << 16); }

// Row of the cache that holds position p of sequence s: (page * heads + head) * page size + slot, or -1.
__device__ __forceinline__ long long cache_row(const CacheArgs& c, const SequencesArgs& g, int s, int p) {
  const int column = p >> c.page_shift;
  if (p < 0 || column >= g.width) return -1;
  const unsigned page = (unsigned)g.pages[(long long)s * g.width + column];
  if (page >= c.pages) return -1;
  return (((long long)page * c.kv_heads) << c.page_shift) + (p & ((1 << c.page_shift) - 1));
}

}  // namespace nimble
#endif
