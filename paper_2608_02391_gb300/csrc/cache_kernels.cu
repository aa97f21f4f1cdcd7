// Pages of a key-value cache: growing, writing, forking, freeing, moving together and copying.
//
// Which page goes where is decided by one block (the free pages in ascending order against the
// list's needs, by prefix sums), so that the same calls give the same pages; what has to be
// copied then is copied by as many blocks as fill the GPU.  The plan is bound by latency (2 us a
// launch in a graph), the copies by HBM.
#include "answer.h"

namespace copes {

__device__ unsigned g_cache_error;
static std::atomic<bool> g_used{false};
__device__ __forceinline__ void flag_error(unsigned bit) { atomicOr(&g_cache_error, bit); }

constexpr int kPlanThreads = 1024;

// The kernels are launched while the one before them on the stream ends, and wait here for all it
// wrote, so that a launch's own time is hidden (fork, grow, append and free of 256 rollouts among three
// copies of the tables: 107 us, 114 without); the next may come as soon as all blocks are here.
__device__ __forceinline__ void after_the_last() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Exclusive prefix sum of v over the block of kPlanThreads and the block's total.  `s` holds 32 ints, one
// for each warp.
__device__ __forceinline__ int block_scan(int v, int *s, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // s may still be read by a previous scan
  if (lane == 31) s[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int w = s[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, w, d);
      if (lane >= d) w += y;
    }
    s[lane] = w;
  }
  __syncthreads();
  *total = s[31];
  return x - v + (warp ? s[warp - 1] : 0);
}

// Writes the pages of [begin, end) that are in use (or free) to list, ascending, and stops after the
// round that finds the most-th; returns how many it found.  Bound by the latency of a round's scan,
// so a thread looks at 8 pages a round: a grow and a free in a pool of 30,000 pages, 29,000 of them
// in use, 13.6 us (one page a round: 22.1), of 1,000 pages 8.4 (7.9).
__device__ __forceinline__ int list_pages(const Cache &c, int begin, int end, bool in_use, int most, int32_t *list, int *s_scan) {
  constexpr int kEach = 8;
  int found = 0;
  for (int base = begin; base < end && found < most; base += kPlanThreads * kEach) {
    const int first = base + (int)threadIdx.x * kEach;
    unsigned mine = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (first + e < end) mine |= (unsigned)((c.refs[first + e] != 0) == in_use) << e;
    int sum, at = found + block_scan(__popc(mine), s_scan, &sum);
    for (; mine; mine &= mine - 1, ++at)
      if (at < most) list[at] = first + __ffs(mine) - 1;
    found += sum;
  }
  return found;
}

__device__ __forceinline__ int pages_of(int tokens, int page_size) {
  return tokens / page_size + (tokens % page_size != 0);
}

// Grow and fork: what every listed slot needs, checked, and the lowest free pages given out.
template <bool kFork>
__global__ void __launch_bounds__(kPlanThreads) cache_plan_kernel(Cache c, const int32_t *slots, const int32_t *parents,
                                                                  const int32_t *add, int add_all, int n, int32_t *ws) {
  __shared__ int s_scan[32];
  __shared__ unsigned s_bad;
  after_the_last();
  const int tid = threadIdx.x;
  int32_t *first = ws + kPlanHeader;       // rank of slot i's first new page
  int32_t *mark = first + c.n_slots;       // by slot: its place in the list
  int32_t *fresh = plan_pages(c, ws);      // the free pages given out, ascending
  if (tid == 0) s_bad = 0;
  for (int i = tid; i < n; i += kPlanThreads)
    if ((unsigned)slots[i] < (unsigned)c.n_slots) mark[slots[i]] = -1;
  if (kFork)
    for (int i = tid; i < n; i += kPlanThreads)
      if ((unsigned)parents[i] < (unsigned)c.n_slots) mark[parents[i]] = -1;
  __syncthreads();

  int total = 0;
  for (int base = 0; base < n; base += kPlanThreads) {
    const int i = base + tid;
    int need = 0, source = -1;
    if (i < n) {
      const int slot = slots[i];
      bool ok = (unsigned)slot < (unsigned)c.n_slots && atomicCAS(&mark[slot], -1, i) == -1;
      if (kFork) {
        const int parent = parents[i];
        ok = ok && (unsigned)parent < (unsigned)c.n_slots && slot_tokens(c, slot) == 0;
        const int tokens = ok ? slot_tokens(c, parent) : 0;
        need = tokens % c.page_size != 0;
        if (need) source = c.table[(int64_t)parent * c.table_width + tokens / c.page_size];
      } else if (ok) {
        const int more = add ? add[i] : add_all;
        const int64_t now = (int64_t)slot_tokens(c, slot) + more;
        ok = more >= 0 && now <= (int64_t)c.table_width * c.page_size;
        if (ok) need = pages_of((int)now, c.page_size) - pages_of(slot_tokens(c, slot), c.page_size);
      }
      if (!ok) atomicOr(&s_bad, kErrCacheId);
    }
    int sum;
    const int at = block_scan(need, s_scan, &sum);
    if (i < n) first[i] = total + at;
    if (kFork && need && total + at < c.n_pages) fresh[c.n_pages + total + at] = source;  // the page to copy
    total += sum;
  }
  __syncthreads();
  if (kFork)  // a child's table is written while the parents' are read
    for (int i = tid; i < n; i += kPlanThreads)
      if ((unsigned)parents[i] < (unsigned)c.n_slots && mark[parents[i]] != -1) atomicOr(&s_bad, kErrCacheId);
  __syncthreads();
  if (s_bad) {
    if (tid == 0) {
      ws[kPlanDone] = 0;
      flag_error(s_bad);
    }
    return;
  }
  const int found = list_pages(c, 0, c.n_pages, false, total, fresh, s_scan);
  if (found < total) {
    if (tid == 0) {
      ws[kPlanDone] = 0;
      flag_error(kErrCacheFull);
    }
    return;
  }
  __syncthreads();  // fresh and first, for every thread
  for (int r = tid; r < total; r += kPlanThreads) {
    const int page = fresh[r];
    c.refs[page] = 1;
    if (kFork) continue;  // the copy's blocks write the children's tables
    int lo = 0, hi = n - 1;  // the last slot whose first page's rank is at most r
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    const int slot = slots[lo];
    c.table[(int64_t)slot * c.table_width + pages_of(slot_tokens(c, slot), c.page_size) + (r - first[lo])] = page;
  }
  __syncthreads();  // lengths are read above
  for (int i = tid; i < n; i += kPlanThreads)
    c.length[slots[i]] = kFork ? slot_tokens(c, parents[i]) : slot_tokens(c, slots[i]) + (add ? add[i] : add_all);
  if (tid == 0) {
    ws[kPlanDone] = 1;
    ws[kPlanTotal] = total;
    ws[kPlanJob] = 0;
  }
}

// A job is 32 KB of a page's copy: 8 pieces of 16 bytes of each thread, all on their way at once.
constexpr int kCopyThreads = 256, kJobPieces = 8 * kCopyThreads;
struct Job {
  int4 v[8];
  __device__ __forceinline__ void load(const Cache &c, int page, int64_t begin) {
    const int4 *at = reinterpret_cast<const int4 *>(c.pool + (uint64_t)page * c.page_bytes);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t i = begin + u * kCopyThreads + threadIdx.x;
      if (i < (int64_t)(c.page_bytes / 16)) v[u] = at[i];
    }
  }
  __device__ __forceinline__ void store(const Cache &c, int page, int64_t begin) const {
    int4 *at = reinterpret_cast<int4 *>(c.pool + (uint64_t)page * c.page_bytes);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t i = begin + u * kCopyThreads + threadIdx.x;
      if (i < (int64_t)(c.page_bytes / 16)) at[i] = v[u];
    }
  }
};
__host__ __device__ inline int64_t jobs_of(const Cache &c) { return (int64_t)(c.page_bytes / 16 + kJobPieces - 1) / kJobPieces; }

// Copies page from[r] to page to[r], r < n, in jobs that the blocks take one after the other: a block's
// first has its own number, the later ones are counted by *taken and asked for while a job is loaded.
// SMs differ by a tenth in the rate at which they reach HBM, so equal shares wait for the slowest: a
// fork with 256 copies of 2.4 MB pages to as many others took 203 us in shares, 185 so.  (A block of its own
// for each job: 186, and a fork without copies 22 us instead of 9.)
__device__ __forceinline__ void copy_pages(const Cache &c, const int32_t *to, const int32_t *from, int n, int32_t *taken) {
  __shared__ int64_t s_next[2];
  const int64_t parts = jobs_of(c), jobs = parts * n;
  int64_t job = blockIdx.x;
  if (job >= jobs) return;
  int64_t begin = job % parts * kJobPieces;
  int source = from[job / parts], target = to[job / parts];
  for (int turn = 0;; turn ^= 1) {
    Job data;
    const bool ok = (unsigned)source < (unsigned)c.n_pages;
    if (ok) data.load(c, source, begin);
    else if (threadIdx.x == 0) flag_error(kErrCacheId);
    const int target_now = target;
    const int64_t begin_now = begin;
    job = jobs;
    if (jobs > gridDim.x) {
      if (threadIdx.x == 0) s_next[turn] = (int64_t)gridDim.x + atomicAdd(reinterpret_cast<unsigned *>(taken), 1u);
      __syncthreads();
      job = s_next[turn];
      if (job < jobs) {
        begin = job % parts * kJobPieces;
        source = from[job / parts];
        target = to[job / parts];
      }
    }
    if (ok) data.store(c, target_now, begin_now);
    if (job >= jobs) return;
  }
}

// Children's tables and the shared pages' refs, then the copies of partly filled pages, which are read
// from L2 after a parent's first child, so that stores bound it: 240 copies of 2.4 MB pages in 88 us,
// 6.4 TB/s.
__global__ void __launch_bounds__(kCopyThreads, 4) fork_copy_kernel(Cache c, const int32_t *parents, const int32_t *children, int n,
                                                        int32_t *ws) {
  after_the_last();
  if (!ws[kPlanDone]) return;
  const int32_t *first = ws + kPlanHeader, *to = plan_pages(c, ws);
  const int spans = (c.table_width - 1) / blockDim.x + 1;  // of a table, an entry for each thread
  for (int64_t u = blockIdx.x; u < (int64_t)n * spans; u += gridDim.x) {
    const int i = (int)(u / spans), j = (int)(u % spans) * blockDim.x + threadIdx.x;
    const int tokens = slot_tokens(c, parents[i]), full = tokens / c.page_size;
    int32_t *entry = c.table + (int64_t)children[i] * c.table_width + j;
    if (j == full && tokens % c.page_size) *entry = to[first[i]];
    if (j >= full) continue;
    const int page = c.table[(int64_t)parents[i] * c.table_width + j];
    *entry = page;
    if ((unsigned)page < (unsigned)c.n_pages) atomicAdd(&c.refs[page], 1);
    else flag_error(kErrCacheId);
  }
  copy_pages(c, to, to + c.n_pages, ws[kPlanTotal], ws + kPlanJob);
}

// One block per slot.  The exchange of the length makes one of a slot's blocks the one that frees it.
__global__ void __launch_bounds__(256) cache_free_kernel(Cache c, const int32_t *slots) {
  __shared__ int s_tokens;
  after_the_last();
  const int slot = slots[blockIdx.x];
  if ((unsigned)slot >= (unsigned)c.n_slots) {
    if (threadIdx.x == 0) flag_error(kErrCacheId);
    return;
  }
  if (threadIdx.x == 0) {
    const int len = atomicExch(&c.length[slot], 0), most = c.table_width * c.page_size;
    s_tokens = len < 0 ? 0 : (len < most ? len : most);
  }
  __syncthreads();
  int32_t *row = c.table + (int64_t)slot * c.table_width;
  for (int j = threadIdx.x; j < pages_of(s_tokens, c.page_size); j += blockDim.x) {
    const int page = row[j];
    row[j] = -1;
    if ((unsigned)page < (unsigned)c.n_pages) atomicSub(&c.refs[page], 1);
    else flag_error(kErrCacheId);
  }
}

// Compact: counts the pages in use (U) and pairs those at U and above with the free ids below.
// ws: to[r] and from[r] of move r (the list of fresh pages' place and the one after it).
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(Cache c, int32_t *counts, int32_t *ws) {
  __shared__ int s_scan[32];
  after_the_last();
  const int tid = threadIdx.x;
  int32_t *to = plan_pages(c, ws), *from = to + c.n_pages;
  int mine = 0, used;
  for (int p = tid; p < c.n_pages; p += kPlanThreads) mine += c.refs[p] != 0;
  block_scan(mine, s_scan, &used);
  list_pages(c, 0, used, false, used, to, s_scan);
  const int movers = list_pages(c, used, c.n_pages, true, c.n_pages, from, s_scan);
  __syncthreads();
  for (int r = tid; r < movers; r += kPlanThreads) {  // as many holes as movers
    c.refs[to[r]] = c.refs[from[r]];
    c.refs[from[r]] = 0;
  }
  if (tid == 0) {
    ws[kPlanTotal] = movers;
    ws[kPlanJob] = 0;
    if (counts) {
      counts[0] = used;
      counts[1] = movers;
    }
  }
}

// The tables' new ids and the moves' copies.  Bound by
// HBM: 369 pages of 2.4 MB, 1.74 GB read and written, in 253 us, 6.9 TB/s (a plain copy: 6.8).
__global__ void __launch_bounds__(kCopyThreads, 4) compact_move_kernel(Cache c, int32_t *ws) {
  after_the_last();
  const int moves = ws[kPlanTotal];
  if (moves == 0) return;
  const int32_t *to = plan_pages(c, ws), *from = to + c.n_pages;
  const int lowest = from[0];  // the moves' sources ascend
  for (int slot = blockIdx.x; slot < c.n_slots; slot += gridDim.x) {
    int32_t *row = c.table + (int64_t)slot * c.table_width;
    const int pages = pages_of(slot_tokens(c, slot), c.page_size);
    for (int j = threadIdx.x; j < pages; j += blockDim.x) {
      const int page = row[j];
      if (page < lowest) continue;
      int lo = 0, hi = moves - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (from[mid] < page) lo = mid + 1;
        else hi = mid;
      }
      if (from[lo] == page) row[j] = to[lo];
    }
  }
  copy_pages(c, to, from, moves, ws + kPlanJob);
}

// A block for each job, as far as a grid goes: 255 copies of one page of 2.4 MB in 82 us, 7.4 TB/s of
// stores.
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(Cache c, const int32_t *src, const int32_t *dst, int n) {
  after_the_last();
  const int64_t parts = jobs_of(c);
  for (int64_t job = blockIdx.x; job < parts * n; job += gridDim.x) {
    const int64_t i = job / parts, begin = job % parts * kJobPieces;
    const int from = src[i], to = dst[i];
    if ((unsigned)from >= (unsigned)c.n_pages || (unsigned)to >= (unsigned)c.n_pages) {
      if (threadIdx.x == 0) flag_error(kErrCacheId);
      continue;
    }
    Job data;
    data.load(c, from, begin);
    data.store(c, to, begin);
  }
}

// A warp per (row, key-value head, key or value).
template <typename T>
__global__ void __launch_bounds__(256) append_kernel(Cache c, int layer, const int32_t *slots, const int32_t *position,
                                                     int n, const T *k, int64_t k_row, int64_t k_head, const T *v,
                                                     int64_t v_row, int64_t v_head) {
  after_the_last();
  const int64_t job = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (job >= (int64_t)n * c.n_kv_heads * 2) return;
  const int which = (int)(job & 1), h = (int)((job >> 1) % c.n_kv_heads), i = (int)((job >> 1) / c.n_kv_heads);
  const int slot = slots ? slots[i] : i;
  bool ok = (unsigned)slot < (unsigned)c.n_slots;
  int page = 0, t = 0;
  if (ok) {
    const int tokens = slot_tokens(c, slot);
    t = position ? position[i] : tokens - 1;
    ok = t >= 0 && t < tokens;
    if (ok) page = c.table[(int64_t)slot * c.table_width + t / c.page_size];
    ok = ok && (unsigned)page < (unsigned)c.n_pages;
  }
  if (!ok) {
    if (lane == 0) flag_error(kErrCacheId);
    return;
  }
  const T *from = which ? v + i * v_row + h * v_head : k + i * k_row + h * k_head;
  T *to = reinterpret_cast<T *>(c.pool + (uint64_t)page * c.page_bytes) + (uint64_t)layer * c.layer_elems +
          (uint64_t)(which * c.n_kv_heads + h) * c.head_elems + (uint64_t)(t % c.page_size) * c.head_dim;
  for (int d = lane; d < c.head_dim; d += 32) to[d] = from[d];
}

// Launches a kernel that begins with after_the_last().
template <typename... Params, typename... Args>
static cudaError_t launch_after(unsigned blocks, unsigned threads, cudaStream_t s, void (*kernel)(Params...), Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

cudaError_t launch_cache_grow(const Cache &c, const int32_t *slots, int n, const int32_t *add, int add_all, int32_t *ws,
                              cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  g_used = true;
  return launch_after(1, kPlanThreads, s, cache_plan_kernel<false>, c, slots, nullptr, add, add_all, n, ws);
}

// What the GPU runs at once with 64 registers a thread.  (Five blocks an SM: 131 us where four take 97.)
constexpr int kCopyBlocks = 152 * 4;

cudaError_t launch_cache_fork(const Cache &c, const int32_t *parents, const int32_t *children, int n, int32_t *ws,
                              cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  g_used = true;
  const cudaError_t e = launch_after(1, kPlanThreads, s, cache_plan_kernel<true>, c, children, parents, nullptr, 0, n, ws);
  if (e != cudaSuccess) return e;
  const int64_t parts = jobs_of(c), spans = (c.table_width - 1) / kCopyThreads + 1;
  const int64_t jobs = (parts > spans ? parts : spans) * n;
  return launch_after((unsigned)(jobs < kCopyBlocks ? jobs : kCopyBlocks), kCopyThreads, s, fork_copy_kernel, c, parents, children, n,
                      ws);
}

cudaError_t launch_cache_free(const Cache &c, const int32_t *slots, int n, cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  g_used = true;
  return launch_after(n, 256, s, cache_free_kernel, c, slots);
}

cudaError_t launch_cache_compact(const Cache &c, int32_t *counts, int32_t *ws, cudaStream_t s) {
  g_used = true;
  const cudaError_t e = launch_after(1, kPlanThreads, s, compact_plan_kernel, c, counts, ws);
  if (e != cudaSuccess) return e;
  return launch_after(kCopyBlocks, kCopyThreads, s, compact_move_kernel, c, ws);
}

cudaError_t launch_cache_copy(const Cache &c, const int32_t *src, const int32_t *dst, int n, cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  g_used = true;
  const int64_t jobs = jobs_of(c) * n;
  return launch_after((unsigned)(jobs < 1 << 30 ? jobs : 1 << 30), kCopyThreads, s, copy_pages_kernel, c, src, dst, n);
}

cudaError_t launch_cache_append(const Cache &c, int layer, const int32_t *slots, const int32_t *position, int n,
                                const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                                int64_t v_head, cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  g_used = true;
  const unsigned blocks = (unsigned)(((int64_t)n * c.n_kv_heads * 2 + 7) / 8);
  if (c.elem == 2)
    return launch_after(blocks, 256, s, append_kernel<uint16_t>, c, layer, slots, position, n, (const uint16_t *)k, k_row,
                        k_head, (const uint16_t *)v, v_row, v_head);
  return launch_after(blocks, 256, s, append_kernel<uint32_t>, c, layer, slots, position, n, (const uint32_t *)k, k_row,
                      k_head, (const uint32_t *)v, v_row, v_head);
}

// Read only once a kernel of this file was launched: copes_check of a program without a cache
// takes as long as before.
unsigned read_and_clear_cache_errors() {
  if (!g_used) return 0;
  unsigned v = 0, zero = 0;
  cudaMemcpyFromSymbol(&v, g_cache_error, sizeof(v));
  if (v) cudaMemcpyToSymbol(g_cache_error, &zero, sizeof(zero));
  return v;
}

}  // namespace copes
