// Device entry point of attention over a paged cache (kernels: paged_tokens_kernel.h, paged_chunks_kernel.h; the division of the work: paged_work.h).
#include <hip/hip_runtime.h>

#include <cmath>

#include "paged_chunks_kernel.h"
#include "paged_tokens_kernel.h"

namespace nimble {

int check_rows(const void* p, int64_t stride, int64_t heads, int64_t D, const char* what);  // (cache_kernels.hip)

template <int D>
static void launch_paged(const PagedArgs& g, const nimble_paged_plan& p, bool int8, hipStream_t stream) {
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(p.grid), dim3(p.block), 0, stream, g); };
  auto join = [&](auto kernel) {
    if (p.parts) hipLaunchKernelGGL(kernel, dim3(p.join_grid[0], p.join_grid[1]), dim3(256), 0, stream, g);
  };
  if (p.kernel == NIMBLE_PAGED_CHUNKS) {
    if (int8) launch(paged_chunks_kernel<D, true>);
    else launch(paged_chunks_kernel<D, false>);
    join(paged_join_kernel<128, D>);
  } else {
    constexpr int kWide = D == 128 ? 4 : 8;  // (of bf16: what the LDS holds)
    if (p.block == 512) {  // (nothing is cut)
      if (int8) launch(paged_tokens_kernel<D, true, 8, false>);
      else launch(paged_tokens_kernel<D, false, kWide, false>);
    } else if (p.parts) {
      if (int8) launch(paged_tokens_kernel<D, true, 4, true>);
      else launch(paged_tokens_kernel<D, false, 4, true>);
    } else {
      if (int8) launch(paged_tokens_kernel<D, true, 4, false>);
      else launch(paged_tokens_kernel<D, false, 4, false>);
    }
    join(paged_join_kernel<16, D>);
  }
}

}  // namespace nimble

using namespace nimble;

extern "C" {

int nimble_paged_attention_dyn(const void* q, int64_t q_stride, const nimble_cache* cache, const nimble_sequences* seqs, void* o,
                               int64_t heads, float alpha, int64_t window, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  int rc = check_cache(cache);
  if (rc == NIMBLE_OK) rc = check_sequences(seqs, cache->page);
  if (rc != NIMBLE_OK) return rc;
  if (!(alpha > 0) || !std::isfinite(alpha)) return fail(NIMBLE_ERR_ARG, "paged_attention: alpha = %g, more than 0 needed", (double)alpha);
  nimble_paged_plan p;
  rc = nimble_paged_attention_plan_of(seqs->rows, seqs->count, seqs->width, heads, cache->kv_heads, cache->page, cache->D, cache->dtype, window, &p);
  if (rc != NIMBLE_OK) return rc;
  if (seqs->rows == 0 || seqs->count == 0) return NIMBLE_OK;
  rc = check_rows(q, q_stride, heads, cache->D, "paged_attention: q");
  if (rc != NIMBLE_OK) return rc;
  if (!o) return fail(NIMBLE_ERR_NULL, "null tensor pointer");
  if (((uintptr_t)o | (uintptr_t)workspace) & 15) return fail(NIMBLE_ERR_ALIGN, "device pointers must be 16-byte aligned");
  if (p.workspace_bytes && (!workspace || workspace_bytes < p.workspace_bytes))
    return fail(NIMBLE_ERR_WORKSPACE, "paged_attention: workspace of %llu bytes needed", (unsigned long long)p.workspace_bytes);
  const auto [ck, cv, cks, cvs] = cache_extents(*cache);
  const auto [offsets, lengths, pages] = sequences_extents(*seqs);
  const int64_t row = heads * cache->D;
  rc = check_apart("paged_attention", {extent("out", o, seqs->rows, row, row), extent("the workspace", workspace, (int64_t)p.workspace_bytes)},
                   {extent("q", q, seqs->rows, row, q_stride), ck, cv, cks, cvs, offsets, lengths, pages});
  if (rc != NIMBLE_OK) return rc;
  PagedArgs g{};
  set_extents(g, *cache, *seqs, heads, window);
  set_parts(g, p, cache->D, workspace);
  g.q = (const uint16_t*)q;
  g.o = (uint16_t*)o;
  g.q_stride = q_stride;
  g.a2 = alpha * 1.4426950408889634f;
  if (!std::isfinite(g.a2)) return fail(NIMBLE_ERR_ARG, "paged_attention: alpha = %g is too large", (double)alpha);
  // Past the caches where each key is read by one workgroup and the page table has room for more than 8 MB: what a layer finds in memory, other
  // layers' caches having been there in between, comes sooner (32 MB 16.7 -> 15.4 us, 256 MB 56.3 -> 49.8), what it finds in the memory-side
  // cache, alone over and over, later (128 MB 33.6 -> 33.0, 34.3 -> 37.3, 256 MB 50.3 -> 53); a short sequence of one token 7.8 -> 8.6.
  g.once = p.kernel == NIMBLE_PAGED_TOKENS && seqs->rows * g.group <= p.rows * seqs->count &&
           (double)seqs->count * seqs->width * cache->page * cache->kv_heads * cache->D * (cache->dtype == NIMBLE_I8 ? 2 : 4) > 8e6;
  if (cache->D == 64)
    launch_paged<64>(g, p, cache->dtype == NIMBLE_I8, (hipStream_t)stream);
  else
    launch_paged<128>(g, p, cache->dtype == NIMBLE_I8, (hipStream_t)stream);
  return check_hip_launch("paged attention kernel launch");
}

}  // extern "C"
