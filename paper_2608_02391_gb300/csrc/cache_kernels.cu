// Pages of a key-value cache: growing, writing, forking, freeing, moving together and copying.
//
// Which page goes where is decided by one block (the free pages in ascending order against the
// list's needs, by prefix sums), so that the same calls give the same pages; what has to be
// copied then is copied by as many blocks as fill the GPU.  The plan is bound by latency (2 us a
// launch in a graph), the copies by HBM.
#include <cuda_fp16.h>

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

// Where the token of a row of append or read is: its page and place there, false (and reported) where there is none.
__device__ __forceinline__ bool find_token(const Cache &c, const int32_t *slots, const int32_t *position, int i, int &page, int &place) {
  const int slot = slots ? slots[i] : i;
  if ((unsigned)slot >= (unsigned)c.n_slots) return false;
  const int tokens = slot_tokens(c, slot), t = position ? position[i] : tokens - 1;
  if (t < 0 || t >= tokens) return false;
  page = c.table[(int64_t)slot * c.table_width + t / c.page_size];
  place = t % c.page_size;
  return (unsigned)page < (unsigned)c.n_pages;
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
  int page, place;
  if (!find_token(c, slots, position, i, page, place)) {
    if (lane == 0) flag_error(kErrCacheId);
    return;
  }
  const T *from = which ? v + i * v_row + h * v_head : k + i * k_row + h * k_head;
  T *to = reinterpret_cast<T *>(c.pool + (uint64_t)page * c.page_bytes) + (uint64_t)layer * c.layer_elems +
          (uint64_t)(which * c.n_kv_heads + h) * c.head_elems + (uint64_t)place * c.head_dim;
  for (int d = lane; d < c.head_dim; d += 32) to[d] = from[d];
}

// A token's key or value in memory of the caller's.
struct Rows {
  uint16_t *at;
  int64_t row, head;
};

// 8 bits.  A team of lanes, a power of two of at least head_dim / 8, for each (row, key or value, key-value head), 8
// values a lane.  The row's unit is the power of two that brings its largest finite value into (224, 448]; as codes are
// floats, a power of two costs no precision that a finer factor would keep.  `wide`: all rows are 16-byte aligned.
//
// Where a row's token is takes a chain of three loads, so a block looks up its rows first, all at once, and
// each thread then has kJobs pieces on their way: 32,000 tokens of 8 heads of 128, 197 MB each way, are written and
// read back in 87 us together, 4.5 TB/s (looked up by each team, with one piece of a thread on its way: 174; with two, 157;
// with eight, 121 where four took 110), bound by HBM and by instructions: 148 of a lane to write 8 values and 101 to read
// them, of which unpacking, scaling, converting and packing are some 30; the rest is a piece's place, address and
// predicates and the maximum's shuffles.  A token each of 64 sequences: 5.7 us.
constexpr int kCodeThreads = 256, kJobs = 4;
struct alignas(16) Place {
  char *codes, *power;  // of the token's first head; NULL: no token
};
template <bool kWrite>
__global__ void __launch_bounds__(kCodeThreads) codes_kernel(Cache c, int layer, const int32_t *slots, const int32_t *position, int n,
                                                             Rows k, Rows v, int team, int rows, bool wide) {
  __shared__ Place s_place[kCodeThreads];
  after_the_last();
  const int row0 = blockIdx.x * rows, here = min(rows, n - row0);
  for (int r = threadIdx.x; r < here; r += kCodeThreads) {
    Place p{nullptr, nullptr};
    int page, place;
    if (find_token(c, slots, position, row0 + r, page, place)) {
      char *base = c.pool + (uint64_t)page * c.page_bytes + layer * c.layer_bytes;
      p = Place{base + (uint64_t)place * c.head_dim, base + c.layer_elems + place};
    } else {
      flag_error(kErrCacheId);
    }
    s_place[r] = p;
  }
  __syncthreads();
  const int d = (int)(threadIdx.x & (team - 1)) * 8, teams = kCodeThreads / team, heads = 2 * c.n_kv_heads;
  const int jobs = here * heads, step_rows = teams / heads, step_heads = teams % heads;
  int row = threadIdx.x / team / heads, head = threadIdx.x / team % heads;  // of the next job
  for (int begun = 0; begun < jobs; begun += teams * kJobs) {
    uint32_t w[kJobs][4];  // 8 values of bf16
    uint16_t *outside[kJobs];
    uint2 *codes[kJobs];
    uint8_t *power[kJobs];
    uint2 held[kJobs];
    uint32_t held_power[kJobs];
#pragma unroll
    for (int u = 0; u < kJobs; ++u) {
      outside[u] = nullptr;
      codes[u] = nullptr;
      if (row < here && d < c.head_dim) {
        // (A reference to one of the two would make the kernel's parameters an array in memory.)
        const bool value = head >= c.n_kv_heads;
        outside[u] = value ? v.at + (row0 + row) * v.row + (head - c.n_kv_heads) * v.head + d : k.at + (row0 + row) * k.row + head * k.head + d;
        const Place at = s_place[row];
        if (at.codes) {
          codes[u] = reinterpret_cast<uint2 *>(at.codes + (uint64_t)head * c.head_elems + d);
          power[u] = reinterpret_cast<uint8_t *>(at.power + (uint64_t)head * c.page_size);
        }
      }
      row += step_rows;
      head += step_heads;
      if (head >= heads) {
        head -= heads;
        ++row;
      }
      if constexpr (kWrite) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[u][e] = 0;
        if (codes[u] && wide) {
          const uint4 x = *reinterpret_cast<const uint4 *>(outside[u]);
          w[u][0] = x.x, w[u][1] = x.y, w[u][2] = x.z, w[u][3] = x.w;
        } else if (codes[u]) {
#pragma unroll
          for (int e = 0; e < 4; ++e) w[u][e] = outside[u][2 * e] | (uint32_t)outside[u][2 * e + 1] << 16;
        }
      } else {
        held[u] = make_uint2(0, 0);
        held_power[u] = 127;
        if (codes[u]) {
          held[u] = *codes[u];
          held_power[u] = *power[u];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kJobs; ++u) {
      if constexpr (kWrite) {
        uint32_t two = 0;  // the largest, as bits of bf16, of even and of odd ones
#pragma unroll
        for (int e = 0; e < 4; ++e) two = __vmaxu2(two, w[u][e] & 0x7FFF7FFFu);
        uint32_t most = max(two & 0xFFFFu, two >> 16);
        const bool finite = most < 0x7F80u;
        if (!finite) {
          most = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t x = w[u][e / 2] >> 16 * (e & 1) & 0x7FFFu;
            if (x < 0x7F80u) most = max(most, x);
            else w[u][e / 2] |= 0x7FFFu << 16 * (e & 1);  // the type has no infinity
          }
        }
        for (int s = team >> 1; s; s >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, s));
        // 127 more than the exponent e: 448 is 1.75 2^8
        const int biased = max((int)(most >> 7) - 8 + ((most & 0x7Fu) > 0x60u), 1);
        const float over = __uint_as_float((uint32_t)(254 - biased) << 23);
        if (!codes[u]) continue;
        uint32_t pair[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float lo = __uint_as_float(w[u][e] << 16) * over, hi = __uint_as_float(w[u][e] & 0xFFFF0000u) * over;
          uint16_t code;
          asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(code) : "f"(hi), "f"(lo));
          pair[e] = code;
        }
        *codes[u] = make_uint2(pair[0] | pair[1] << 16, pair[2] | pair[3] << 16);
        if (d == 0) *power[u] = (uint8_t)biased;
      } else {
        if (!outside[u]) continue;
        const float unit = __uint_as_float(held_power[u] << 23);
        uint32_t out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint16_t two = (uint16_t)((e < 2 ? held[u].x : held[u].y) >> 16 * (e & 1));
          uint32_t both;
          asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(both) : "h"(two));
          const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&both));
          const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * unit, f.y * unit);
          out[e] = *reinterpret_cast<const uint32_t *>(&b);
        }
        if (wide) {
          *reinterpret_cast<uint4 *>(outside[u]) = make_uint4(out[0], out[1], out[2], out[3]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) outside[u][e] = (uint16_t)(out[e / 2] >> 16 * (e & 1));
        }
      }
    }
  }
}

// A warp per (row, key-value head, key or value), as append_kernel.
template <typename T>
__global__ void __launch_bounds__(256) read_kernel(Cache c, int layer, const int32_t *slots, const int32_t *position, int n, T *k,
                                                   int64_t k_row, int64_t k_head, T *v, int64_t v_row, int64_t v_head) {
  after_the_last();
  const int64_t job = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (job >= (int64_t)n * c.n_kv_heads * 2) return;
  const int which = (int)(job & 1), h = (int)((job >> 1) % c.n_kv_heads), i = (int)((job >> 1) / c.n_kv_heads);
  T *to = which ? v + i * v_row + h * v_head : k + i * k_row + h * k_head;
  int page, place;
  if (!find_token(c, slots, position, i, page, place)) {
    if (lane == 0) flag_error(kErrCacheId);
    for (int d = lane; d < c.head_dim; d += 32) to[d] = 0;
    return;
  }
  const T *from = reinterpret_cast<const T *>(c.pool + (uint64_t)page * c.page_bytes) + (uint64_t)layer * c.layer_elems +
                  (uint64_t)(which * c.n_kv_heads + h) * c.head_elems + (uint64_t)place * c.head_dim;
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

template <bool kWrite>
static cudaError_t launch_codes(const Cache &c, int layer, const int32_t *slots, const int32_t *position, int n, Rows k, Rows v,
                                cudaStream_t s) {
  int team = 2;
  while (team * 8 < c.head_dim) team *= 2;
  uintptr_t all = 0;
  for (const Rows &r : {k, v}) all |= (uintptr_t)r.at | (uintptr_t)r.row * 2 | (uintptr_t)r.head * 2;
  const int each = (n - 1) / (152 * 4) + 1, rows = each < kCodeThreads ? each : kCodeThreads;  // of a block, of as many as run at once
  return launch_after((n - 1) / rows + 1, kCodeThreads, s, codes_kernel<kWrite>, c, layer, slots, position, n, k, v, team, rows, all % 16 == 0);
}

cudaError_t launch_cache_append(const Cache &c, int layer, const int32_t *slots, const int32_t *position, int n,
                                const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                                int64_t v_head, cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  g_used = true;
  if (c.elem == 1)
    return launch_codes<true>(c, layer, slots, position, n, {(uint16_t *)k, k_row, k_head}, {(uint16_t *)v, v_row, v_head}, s);
  const unsigned blocks = (unsigned)(((int64_t)n * c.n_kv_heads * 2 + 7) / 8);
  if (c.elem == 2)
    return launch_after(blocks, 256, s, append_kernel<uint16_t>, c, layer, slots, position, n, (const uint16_t *)k, k_row,
                        k_head, (const uint16_t *)v, v_row, v_head);
  return launch_after(blocks, 256, s, append_kernel<uint32_t>, c, layer, slots, position, n, (const uint32_t *)k, k_row,
                      k_head, (const uint32_t *)v, v_row, v_head);
}

cudaError_t launch_cache_read(const Cache &c, int layer, const int32_t *slots, const int32_t *position, int n, void *k,
                              int64_t k_row, int64_t k_head, void *v, int64_t v_row, int64_t v_head, cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  g_used = true;
  if (c.elem == 1)
    return launch_codes<false>(c, layer, slots, position, n, {(uint16_t *)k, k_row, k_head}, {(uint16_t *)v, v_row, v_head}, s);
  const unsigned blocks = (unsigned)(((int64_t)n * c.n_kv_heads * 2 + 7) / 8);
  if (c.elem == 2)
    return launch_after(blocks, 256, s, read_kernel<uint16_t>, c, layer, slots, position, n, (uint16_t *)k, k_row, k_head,
                        (uint16_t *)v, v_row, v_head);
  return launch_after(blocks, 256, s, read_kernel<uint32_t>, c, layer, slots, position, n, (uint32_t *)k, k_row, k_head,
                      (uint32_t *)v, v_row, v_head);
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
