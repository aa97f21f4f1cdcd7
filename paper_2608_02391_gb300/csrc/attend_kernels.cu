// Attention of one new token per sequence over a paged key-value cache.
#include <math.h>

#include "answer.h"

namespace copes {

__device__ unsigned g_attend_error;
static std::atomic<bool> g_used{false};
__device__ __forceinline__ void flag_error(unsigned bit) { atomicOr(&g_attend_error, bit); }

constexpr int kAttendThreads = 128;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float x, float *to) { *to = x; }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16 *to) { *to = __float2bfloat16_rn(x); }

// A block per (row, query head): a chunk of tokens at a time, a thread per token for the scores
// and a thread per value component for the sums, with the running maximum and sum of the softmax.
template <typename T>
__global__ void __launch_bounds__(kAttendThreads) attend_simple_kernel(AttendArgs a) {
  __shared__ float s_q[COPES_MAX_HEAD_DIM], s_p[kAttendThreads], s_red[kAttendThreads];
  __shared__ int s_page[kAttendThreads];
  const Cache &c = a.c;
  const int tid = threadIdx.x, i = blockIdx.x / a.q_heads, h = blockIdx.x % a.q_heads;
  const int g = h / (a.q_heads / c.n_kv_heads), D = c.head_dim;
  const int slot = a.slots ? a.slots[i] : i;
  int tokens = 0;
  if ((unsigned)slot < (unsigned)c.n_slots) tokens = slot_tokens(c, slot);
  else if (tid == 0) flag_error(kErrCacheId);
  const T *q = (const T *)a.q + i * a.q_row + h * a.q_head;
  for (int d = tid; d < D; d += kAttendThreads) s_q[d] = to_float(q[d]) * a.scale;
  float m = -INFINITY, l = 0.0f, o[COPES_MAX_HEAD_DIM / kAttendThreads] = {};
  const uint64_t k_at = (uint64_t)a.layer * c.layer_elems + (uint64_t)g * c.head_elems;
  const uint64_t v_at = k_at + (uint64_t)c.n_kv_heads * c.head_elems;
  for (int base = 0; base < tokens; base += kAttendThreads) {
    const int t = base + tid, here = min(kAttendThreads, tokens - base);
    __syncthreads();
    float s = -INFINITY;
    if (t < tokens) {
      int page = c.table[(int64_t)slot * c.table_width + t / c.page_size];
      if ((unsigned)page >= (unsigned)c.n_pages) {
        flag_error(kErrCacheId);
        page = -1;
      }
      s_page[tid] = page;
      s = 0.0f;
      if (page >= 0) {
        const T *k = (const T *)(c.pool + (uint64_t)page * c.page_bytes) + k_at + (uint64_t)(t % c.page_size) * D;
        for (int d = 0; d < D; ++d) s = fmaf(to_float(k[d]), s_q[d], s);
      }
    }
    s_red[tid] = s;
    __syncthreads();
    float top = m;
    for (int j = 0; j < here; ++j) top = fmaxf(top, s_red[j]);
    const float p = t < tokens ? expf(s - top) : 0.0f, keep = expf(m - top);
    s_p[tid] = p;
    __syncthreads();
    m = top;
    l *= keep;
    for (int j = 0; j < here; ++j) l += s_p[j];
    for (int r = 0, d = tid; d < D; d += kAttendThreads, ++r) {
      float x = o[r] * keep;
      for (int j = 0; j < here; ++j)
        if (s_page[j] >= 0)
          x = fmaf(s_p[j], to_float(((const T *)(c.pool + (uint64_t)s_page[j] * c.page_bytes))[
                                v_at + (uint64_t)((base + j) % c.page_size) * D + d]), x);
      o[r] = x;
    }
  }
  T *out = (T *)a.out + ((int64_t)i * a.q_heads + h) * D;
  for (int r = 0, d = tid; d < D; d += kAttendThreads, ++r) from_float(tokens ? o[r] / l : 0.0f, out + d);
  if (tid == 0 && a.lse) a.lse[(int64_t)i * a.q_heads + h] = tokens ? m + logf(l) : -INFINITY;
}

size_t attend_workspace_bytes(const Cache &, int, int) { return 16; }

cudaError_t launch_paged_attention(int dtype, const AttendArgs &a, void *, cudaStream_t s) {
  if (a.n == 0) return cudaSuccess;
  g_used = true;
  const unsigned blocks = (unsigned)a.n * a.q_heads;
  if (dtype == COPES_BF16) attend_simple_kernel<__nv_bfloat16><<<blocks, kAttendThreads, 0, s>>>(a);
  else attend_simple_kernel<float><<<blocks, kAttendThreads, 0, s>>>(a);
  return cudaGetLastError();
}

unsigned read_and_clear_attend_errors() {
  if (!g_used) return 0;
  unsigned v = 0, zero = 0;
  cudaMemcpyFromSymbol(&v, g_attend_error, sizeof(v));
  if (v) cudaMemcpyToSymbol(g_attend_error, &zero, sizeof(zero));
  return v;
}

}  // namespace copes
