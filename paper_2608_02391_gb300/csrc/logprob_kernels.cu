// Log probabilities of given tokens, with entropy and top alternatives.
#include <math.h>

#include "answer.h"

namespace copes {

__device__ unsigned g_logprob_error;
static std::atomic<bool> g_used{false};
__device__ __forceinline__ void flag_error(unsigned bit) { atomicOr(&g_logprob_error, bit); }

constexpr int kLogprobThreads = 512;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// (value, index) as one number whose order is: larger value first, then lower index.  -0 is 0;
// NaN is above +inf.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t index) {
  uint32_t b = __float_as_uint(x + 0.0f);
  if (x != x) b = 0x7FFFFFFFu;
  b = (b >> 31) ? ~b : b | 0x80000000u;
  return (uint64_t)b << 32 | (uint32_t)~index;
}

template <typename V, typename Op>
__device__ __forceinline__ V block_reduce(V v, Op op, V *s) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < kLogprobThreads / 32; ++w) v = op(v, s[w]);
  return v;
}

// A block per row: the maximum, then the sums, then the alternatives one by one.
template <typename T>
__global__ void __launch_bounds__(kLogprobThreads) logprob_simple_kernel(LogprobArgs a) {
  __shared__ float s_f[kLogprobThreads / 32];
  __shared__ uint64_t s_k[kLogprobThreads / 32];
  const int tid = threadIdx.x, i = blockIdx.x;
  const T *x = (const T *)a.logits + (int64_t)i * a.row;
  const auto add = [](float u, float v) { return u + v; };
  const auto most = [](uint64_t u, uint64_t v) { return u > v ? u : v; };

  uint64_t best = 0;
  float odd = 0.0f;  // NaN where the row holds NaN or +inf
  for (int j = tid; j < a.vocab; j += kLogprobThreads) {
    const float v = to_float(x[j]);
    best = most(best, order_key(v, j));
    if (!(v < INFINITY)) odd = NAN;
  }
  best = block_reduce(best, most, s_k);
  odd = block_reduce(odd, add, s_f);
  const float top = to_float(x[(uint32_t)~(uint32_t)best]);
  const bool empty = top == -INFINITY;
  float sum = 0.0f, weighted = 0.0f;
  for (int j = tid; j < a.vocab && !empty; j += kLogprobThreads) {
    const float away = fmaxf((to_float(x[j]) - top) * a.scale, -1e30f), e = expf(away);
    sum += e;
    weighted = fmaf(e, away, weighted);
  }
  sum = block_reduce(sum, add, s_f);
  weighted = block_reduce(weighted, add, s_f);
  const float log_sum = logf(sum);
  if (tid == 0) {
    const int64_t t = a.target[i];
    float lp = 0.0f;
    if (t >= a.vocab) {
      flag_error(kErrCacheId);
      lp = NAN;
    } else if (t >= 0) {
      lp = empty ? -INFINITY : (to_float(x[t]) - top) * a.scale - log_sum + odd;
    }
    a.logprob[i] = lp;
    if (a.entropy) a.entropy[i] = empty ? 0.0f : log_sum - weighted / sum + odd;
  }
  for (int r = 0; r < a.top; ++r) {
    if (r) {  // the next below the last
      uint64_t next = 0;
      for (int j = tid; j < a.vocab; j += kLogprobThreads) {
        const uint64_t k = order_key(to_float(x[j]), j);
        if (k < best) next = most(next, k);
      }
      best = block_reduce(next, most, s_k);
    }
    if (tid == 0) {
      const uint32_t id = (uint32_t)~(uint32_t)best;
      a.top_ids[(int64_t)i * a.top + r] = id;
      a.top_logprobs[(int64_t)i * a.top + r] = empty ? -INFINITY : (to_float(x[id]) - top) * a.scale - log_sum + odd;
    }
  }
}

cudaError_t launch_token_logprobs(int dtype, const LogprobArgs &a, cudaStream_t s) {
  if (a.n == 0) return cudaSuccess;
  g_used = true;
  if (dtype == COPES_BF16) logprob_simple_kernel<__nv_bfloat16><<<a.n, kLogprobThreads, 0, s>>>(a);
  else logprob_simple_kernel<float><<<a.n, kLogprobThreads, 0, s>>>(a);
  return cudaGetLastError();
}

unsigned read_and_clear_logprob_errors() {
  if (!g_used) return 0;
  unsigned v = 0, zero = 0;
  cudaMemcpyFromSymbol(&v, g_logprob_error, sizeof(v));
  if (v) cudaMemcpyToSymbol(g_logprob_error, &zero, sizeof(zero));
  return v;
}

}  // namespace copes
