// Declarations shared by the kernels that answer with the weights (key-value cache, paged
// attention, token log probabilities) and their host side.
#pragma once

#include <atomic>

#include <cuda_bf16.h>

#include "copes_internal.h"

namespace copes {

// Further device error bits (the first five are in copes_internal.h).
enum : unsigned {
  kErrCacheId = 32u,   // a slot, page, token or target id outside its range, or named twice
  kErrCacheFull = 64u  // more pages asked for than are free
};

// A copes_kv_cache as the kernels take it.
struct Cache {
  char *pool;
  int32_t *table, *length, *refs;
  uint64_t page_bytes;   // of all layers
  uint64_t layer_elems;  // 2 * n_kv_heads * page_size * head_dim
  uint32_t head_elems;   // page_size * head_dim (below 2^31: page_size is)
  int elem;              // bytes of an element
  int n_pages, n_layers, n_kv_heads, page_size, head_dim, n_slots, table_width;
};

// The tokens of a slot, whatever its length entry holds.
__device__ __forceinline__ int slot_tokens(const Cache &c, int slot) {
  const int len = c.length[slot], most = c.table_width * c.page_size;
  return len < 0 ? 0 : (len < most ? len : most);
}

// Workspace of the page plans, in int32: a header (kPlan...), by listed slot the rank of its first new
// page, by slot its place in the list, and two lists of pages.
enum { kPlanDone = 0, kPlanTotal = 1, kPlanJob = 2, kPlanHeader = 4 };
inline size_t cache_workspace_ints(int n_pages, int n_slots) {
  return (size_t)kPlanHeader + 2 * (size_t)n_slots + 2 * (size_t)n_pages;
}
template <typename Int>
__device__ __forceinline__ Int *plan_pages(const Cache &c, Int *ws) {
  return ws + kPlanHeader + 2 * (size_t)c.n_slots;
}

cudaError_t launch_cache_grow(const Cache &c, const int32_t *slots, int n, const int32_t *add, int add_all,
                              int32_t *ws, cudaStream_t s);
cudaError_t launch_cache_append(const Cache &c, int layer, const int32_t *slots, const int32_t *position, int n,
                                const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                                int64_t v_head, cudaStream_t s);
cudaError_t launch_cache_fork(const Cache &c, const int32_t *parents, const int32_t *children, int n, int32_t *ws,
                              cudaStream_t s);
cudaError_t launch_cache_free(const Cache &c, const int32_t *slots, int n, cudaStream_t s);
cudaError_t launch_cache_compact(const Cache &c, int32_t *counts, int32_t *ws, cudaStream_t s);
cudaError_t launch_cache_copy(const Cache &c, const int32_t *src, const int32_t *dst, int n, cudaStream_t s);

struct AttendArgs {
  Cache c;
  int layer, n, q_heads;
  const int32_t *slots;
  const void *q;
  int64_t q_row, q_head;
  float scale;
  void *out;
  float *lse;
};
size_t attend_workspace_bytes(const Cache &c, int n, int q_heads);
cudaError_t launch_paged_attention(int dtype, const AttendArgs &a, void *ws, cudaStream_t s);

struct LogprobArgs {
  const void *logits;
  int64_t row;
  const int64_t *target;
  int n, vocab, top;
  float scale;
  float *logprob, *entropy;
  int64_t *top_ids;
  float *top_logprobs;
};
cudaError_t launch_token_logprobs(int dtype, const LogprobArgs &a, cudaStream_t s);

// Device error words of each translation unit: read and clear (synchronous); 0 without a copy
// where none of its kernels was launched.
unsigned read_and_clear_cache_errors();
unsigned read_and_clear_attend_errors();
unsigned read_and_clear_logprob_errors();

}  // namespace copes
