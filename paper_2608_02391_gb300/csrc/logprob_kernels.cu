// Log probabilities of given tokens, with entropy and top alternatives, from one pass over the
// logits.
//
// With m the row's maximum, y_j = scale (x_j - m) log2 e, s = sum 2^y_j and h = sum y_j 2^y_j:
//   logprob of t = scale (x_t - m) - ln s,   entropy = ln s - ln 2 h / s.
// A warp keeps a running m of what it has read and rescales its sums where that grows by
// g = scale (m' - m) log2 e (h' = 2^-g (h - g s)), so each logit is read once.  y is held at
// kLeast or above, where 2^y is 0: a masked token adds 0 to both sums.  A logit costs
// one exponential and about six more instructions: at 6.8 TB/s of bf16 the exponentials fill
// 75% of the special-function units and the whole half of the issue slots, and HBM bounds it.
//
// The alternatives need no second pass over the row: while it is read, the maximum of every cell
// (a few adjacent 16-byte pieces) is kept in shared memory.  Cells are dealt into 32 groups; the
// k-th largest of the groups' maxima is a bound that k logits at least reach, so only cells that
// reach it hold alternatives.  They are about k to 4 k of 1,024 at most, and are read again, from
// L2.  Their logits that reach the bound are ranked by counting.
//
// A row is read by one block, or, where there are few rows, by a cluster of up to 8 blocks whose
// first joins the others' sums and alternatives through its shared memory.
#include <float.h>
#include <math.h>

#include "answer.h"

namespace copes {

__device__ unsigned g_logprob_error;
static std::atomic<bool> g_used{false};
__device__ __forceinline__ void flag_error(unsigned bit) { atomicOr(&g_logprob_error, bit); }

constexpr unsigned kAll = 0xffffffffu;
constexpr int kThreads_ = 256, kWarps_ = kThreads_ / 32;
constexpr int kCells = 1024;      // of a block's part of a row, at most
constexpr int kCandidates = 512;  // at most, by the fast way
constexpr int kClusterMost = 8;
constexpr int kLoads = 4;         // 16-byte pieces of a lane in one step

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t x, float &a, float &b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// A logit as an integer of the same order.  -0 is 0, and any NaN the largest.
__device__ __forceinline__ int order_of(float x) {
  const int b = __float_as_int(x + 0.0f);
  const int o = b ^ ((b >> 31) & 0x7FFFFFFF);
  return x != x ? 0x7FFFFFFF : o;
}
__device__ __forceinline__ float value_of(int o) { return __int_as_float(o ^ ((o >> 31) & 0x7FFFFFFF)); }
constexpr int kNone = (int)0x80000000;  // below every logit

// A logit and its index as one number: larger logits are larger, then lower indices.  0: none.
__device__ __forceinline__ uint64_t ranked(int order, uint32_t index) {
  return (uint64_t)((uint32_t)order ^ 0x80000000u) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ int order_in(uint64_t r) { return (int)((uint32_t)(r >> 32) ^ 0x80000000u); }
__device__ __forceinline__ uint32_t index_in(uint64_t r) { return ~(uint32_t)r; }

template <typename T>
struct Piece {  // 16 bytes of logits
  static constexpr int kN = 16 / sizeof(T);
  uint32_t r[4];
};
template <typename T>
__device__ __forceinline__ void pair_of(const Piece<T> &p, int i, float &a, float &b) {  // logits 2 i, 2 i + 1
  if constexpr (sizeof(T) == 2) {
    a = __uint_as_float(p.r[i] << 16);
    b = __uint_as_float(p.r[i] & 0xFFFF0000u);
  } else {
    a = __uint_as_float(p.r[2 * i]);
    b = __uint_as_float(p.r[2 * i + 1]);
  }
}
template <typename T>
__device__ __forceinline__ float max_of(const Piece<T> &p) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t m = max_nan_bf16x2(max_nan_bf16x2(p.r[0], p.r[1]), max_nan_bf16x2(p.r[2], p.r[3]));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  } else {
    return max_nan(max_nan(__uint_as_float(p.r[0]), __uint_as_float(p.r[1])),
                   max_nan(__uint_as_float(p.r[2]), __uint_as_float(p.r[3])));
  }
}

// A row in aligned pieces of 16 bytes: piece v holds logits v kN - shift and on; the first and
// the last may hold fewer than kN.
template <typename T>
struct Row {
  const T *x;
  int vocab, shift;
  __device__ Row(const T *row, int n) : x(row), vocab(n), shift((int)(((uintptr_t)row & 15) / sizeof(T))) {}
  __device__ int pieces() const { return (int)(((int64_t)shift + vocab + Piece<T>::kN - 1) / Piece<T>::kN); }
  __device__ int first(int v) const { return v * Piece<T>::kN - shift; }
  // what lies outside the row reads as -inf
  __device__ __forceinline__ Piece<T> load(int v) const {
    Piece<T> p;
    const int j = first(v);
    if (j >= 0 && j + Piece<T>::kN <= vocab) {
      asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(p.r[0]), "=r"(p.r[1]), "=r"(p.r[2]), "=r"(p.r[3]) : "l"(x + j));
      return p;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        uint32_t u = 0xFF80u, w = 0xFF80u;
        if (j + 2 * i >= 0 && j + 2 * i < vocab) u = reinterpret_cast<const uint16_t *>(x)[j + 2 * i];
        if (j + 2 * i + 1 >= 0 && j + 2 * i + 1 < vocab) w = reinterpret_cast<const uint16_t *>(x)[j + 2 * i + 1];
        p.r[i] = u | w << 16;
      } else {
        p.r[i] = j + i >= 0 && j + i < vocab ? reinterpret_cast<const uint32_t *>(x)[j + i] : 0xFF800000u;
      }
    }
    return p;
  }
};

struct Sums {
  float m, s, h;
};

constexpr float kLeast = -16384.0f;

// Sums taken relative to m, wanted relative to M >= m; c is scale log2 e.
__device__ __forceinline__ void rebase(float &s, float &h, float m, float M, float c) {
  const float y = max_nan((m - M) * c, kLeast), f = exp2_fast(y);
  h = f * fmaf(s, y, h);
  s = f * s;
}

__device__ __forceinline__ Sums join(Sums a, Sums b, float c) {
  const float M = max_nan(a.m, b.m);
  rebase(a.s, a.h, a.m, M, c);
  rebase(b.s, b.h, b.m, M, c);
  return {M, a.s + b.s, a.h + b.h};
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
// The address of the cluster's first block's copy of a shared variable.
__device__ __forceinline__ uint32_t in_first(const void *p) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)));
  return r;
}

struct LogprobShared {
  int cell[kCells];                // maxima, as order_of
  uint16_t reached[kCells];        // cells that reach the bound
  uint64_t candidate[kCandidates];
  uint64_t top[COPES_MAX_TOP];
  uint64_t theirs[kClusterMost * COPES_MAX_TOP];  // of the cluster's blocks, in the first
  Sums sums[kClusterMost];
  int group[kWarps_][32];
  Sums warp[kWarps_];
  uint64_t best[kWarps_];
  int n_reached, n_candidates;
};

// top[0 .. k): the k largest of list[0 .. n), 0 past them.  By counting: the numbers differ.
__device__ __forceinline__ void rank_by_counting(const uint64_t *list, int n, int k, uint64_t *top) {
  for (int i = threadIdx.x; i < n; i += kThreads_) {
    const uint64_t mine = list[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += list[j] > mine;
    if (rank < k && mine) top[rank] = mine;
  }
}

// The block's alternatives into sh.top, from the cells' maxima of pieces [v0, v0 + n).
template <typename T>
__device__ void find_top(LogprobShared &sh, const Row<T> &row, int v0, int n, int cell_log, int k) {
  constexpr int N = Piece<T>::kN;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cells = (n + (1 << cell_log) - 1) >> cell_log;
  int best = kNone;
  for (int i = tid; i < cells; i += kThreads_) best = max(best, sh.cell[i]);
  sh.group[warp][lane] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps_; ++w) best = max(best, sh.group[w][lane]);
  int rank = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const int other = __shfl_sync(kAll, best, i);
    rank += other > best || (other == best && i < lane);
  }
  const int bound = __shfl_sync(kAll, best, __ffs(__ballot_sync(kAll, rank == k - 1)) - 1);
  for (int i = tid; i < cells; i += kThreads_)
    if (sh.cell[i] >= bound) sh.reached[atomicAdd(&sh.n_reached, 1)] = (uint16_t)i;
  __syncthreads();
  const int items = sh.n_reached << cell_log;  // a cell's pieces are at most n, cells at most kCells

  // visit(logit's order, its index) for every logit of the cells that reach the bound
  const auto each = [&](auto visit) {
    for (int i = tid; i < items; i += kThreads_) {
      const int v = ((int)sh.reached[i >> cell_log] << cell_log) + (i & ((1 << cell_log) - 1));
      if (v >= n) continue;
      const Piece<T> p = row.load(v0 + v);
      const int j = row.first(v0 + v);
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        float x[2];
        pair_of(p, e, x[0], x[1]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if ((unsigned)(j + 2 * e + u) < (unsigned)row.vocab) visit(order_of(x[u]), (uint32_t)(j + 2 * e + u));
      }
    }
  };
  const auto push = [&](int order, uint32_t index) {
    const int at = atomicAdd(&sh.n_candidates, 1);
    if (at < kCandidates) sh.candidate[at] = ranked(order, index);
  };
  each([&](int order, uint32_t index) {
    if (order >= bound) push(order, index);
  });
  __syncthreads();
  int found = sh.n_candidates;
  if (found > kCandidates) {
    // Many equal the bound (masked tokens where fewer than k are left), or many surpass it (logits
    // in order).  The former: those that surpass it, and the first k that equal it.
    __syncthreads();
    if (tid == 0) sh.n_candidates = 0;
    __syncthreads();
    each([&](int order, uint32_t index) {
      if (order > bound) push(order, index);
    });
    __syncthreads();
    found = sh.n_candidates;
    if (found <= kCandidates - COPES_MAX_TOP) {
      if (warp == 0) {
        int equal = 0;
        for (int v = lane; equal < k && v - lane < n; v += 32) {  // in the order of the indices
          const bool here = v < n && sh.cell[v >> cell_log] >= bound;
          if (!__any_sync(kAll, here)) continue;
          float x[N];
          int j = 0, mine = 0;
          if (here) {
            const Piece<T> p = row.load(v0 + v);
            j = row.first(v0 + v);
#pragma unroll
            for (int e = 0; e < N / 2; ++e) pair_of(p, e, x[2 * e], x[2 * e + 1]);
#pragma unroll
            for (int e = 0; e < N; ++e) mine += (unsigned)(j + e) < (unsigned)row.vocab && order_of(x[e]) == bound;
          }
          int before = mine;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(kAll, before, d);
            if (lane >= d) before += y;
          }
          const int sum = __shfl_sync(kAll, before, 31);
          int at = equal + before - mine;
          if (here) {
#pragma unroll
            for (int e = 0; e < N; ++e)
              if ((unsigned)(j + e) < (unsigned)row.vocab && order_of(x[e]) == bound) {
                if (at < k) sh.candidate[found + at] = ranked(bound, (uint32_t)(j + e));
                ++at;
              }
          }
          equal += sum;
        }
        if (lane == 0) sh.n_candidates = found + min(equal, k);
      }
      __syncthreads();
      found = sh.n_candidates;
    }
  }
  if (found <= kCandidates) {
    rank_by_counting(sh.candidate, found, k, sh.top);
    __syncthreads();
    return;
  }
  uint64_t last = ~0ull;  // one after the other
  for (int r = 0; r < k; ++r) {
    uint64_t next = 0;
    each([&](int order, uint32_t index) {
      const uint64_t key = ranked(order, index);
      if (key < last && key > next) next = key;
    });
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      const uint64_t y = __shfl_xor_sync(kAll, next, d);
      if (y > next) next = y;
    }
    if (lane == 0) sh.best[warp] = next;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps_; ++w)
      if (sh.best[w] > next) next = sh.best[w];
    if (tid == 0) sh.top[r] = next;
    last = next;
    __syncthreads();
  }
}

// Block (or cluster of `parts` blocks) per row; a cell is 2^cell_log pieces.
template <typename T, bool kTop>
__global__ void __launch_bounds__(kThreads_, 4) logprob_kernel(LogprobArgs a, int parts, int cell_log) {
  __shared__ LogprobShared sh;
  constexpr int N = Piece<T>::kN;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int i = blockIdx.x / parts, part = blockIdx.x % parts;
  if (parts > 1) cluster_arrive();
  const Row<T> row((const T *)a.logits + (int64_t)i * a.row, a.vocab);
  const int all = row.pieces();
  const int v0 = (int)((int64_t)all * part / parts), n = (int)((int64_t)all * (part + 1) / parts) - v0;
  const float c = a.scale * 1.44269504088896340736f;
  const int64_t target = a.target[i];
  if (kTop) {
    const int cells = (n + (1 << cell_log) - 1) >> cell_log;
    if (tid < COPES_MAX_TOP) sh.top[tid] = 0;
    if (tid == 0) sh.n_reached = sh.n_candidates = 0;
    if (cell_log > 5)
      for (int j = tid; j < cells; j += kThreads_) sh.cell[j] = kNone;
    __syncthreads();
  }

  Sums t{-FLT_MAX, 0.0f, 0.0f};
  uint64_t s2 = 0, h2 = 0;
  const uint64_t c2 = pack2(c, c);
  constexpr int kStep = kLoads * 32;
  Piece<T> now[kLoads];
  const auto fetch = [&](int base, Piece<T> (&to)[kLoads]) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int v = base + u * 32 + lane;
      if (v < n) {
        to[u] = row.load(v0 + v);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) to[u].r[e] = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
      }
    }
  };
  if (warp * kStep < n) fetch(warp * kStep, now);
  for (int base = warp * kStep; base < n; base += kWarps_ * kStep) {
    Piece<T> next[kLoads];
    if (base + kWarps_ * kStep < n) fetch(base + kWarps_ * kStep, next);
    float most[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) most[u] = max_of(now[u]);
    if (kTop) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int v = base + u * 32 + lane;
        int o = order_of(most[u]);
        if (cell_log >= 5) o = __reduce_max_sync(kAll, o);
        else
          for (int d = 1; d < (1 << cell_log); d <<= 1) o = max(o, __shfl_xor_sync(kAll, o, d));
        if (cell_log > 5) {
          if (lane == 0 && v < n) atomicMax(&sh.cell[v >> cell_log], o);
        } else if ((v & ((1 << cell_log) - 1)) == 0 && v < n) {
          sh.cell[v >> cell_log] = o;
        }
      }
    }
    const float lane_most = max_nan(max_nan(most[0], most[1]), max_nan(most[2], most[3]));
    const float M = max_nan(t.m, value_of(__reduce_max_sync(kAll, order_of(lane_most))));
    if (!(M == t.m)) {  // the same for the whole warp
      float s0, s1, h0, h1;
      unpack2(s2, s0, s1);
      unpack2(h2, h0, h1);
      s0 += s1;
      h0 += h1;
      rebase(s0, h0, t.m, M, c);
      s2 = pack2(s0, 0.0f);
      h2 = pack2(h0, 0.0f);
      t.m = M;
    }
    const uint64_t minus_m = pack2(-t.m, -t.m);
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        float x, y;
        pair_of(now[u], e, x, y);
        float d0, d1;
        unpack2(mul2(add2(pack2(x, y), minus_m), c2), d0, d1);
        d0 = max_nan(d0, kLeast);
        d1 = max_nan(d1, kLeast);
        const uint64_t p = pack2(exp2_fast(d0), exp2_fast(d1));
        s2 = add2(s2, p);
        h2 = fma2(p, pack2(d0, d1), h2);
      }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) now[u] = next[u];
  }
  float odd_s, odd_h;
  unpack2(s2, t.s, odd_s);
  unpack2(h2, t.h, odd_h);
  t.s += odd_s;
  t.h += odd_h;
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    t.s += __shfl_xor_sync(kAll, t.s, d);
    t.h += __shfl_xor_sync(kAll, t.h, d);
  }
  if (lane == 0) sh.warp[warp] = t;
  __syncthreads();
  t = sh.warp[0];
#pragma unroll
  for (int w = 1; w < kWarps_; ++w) t = join(t, sh.warp[w], c);
  if (kTop) find_top(sh, row, v0, n, cell_log, a.top);

  if (parts > 1) {
    cluster_wait();  // the first block has begun
    const uint32_t to = in_first(&sh.sums[part]);
    if (tid < 3)
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4 * tid), "f"(tid == 0 ? t.m : tid == 1 ? t.s : t.h) : "memory");
    if (kTop && tid < a.top)
      asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(in_first(&sh.theirs[part * a.top + tid])), "l"(sh.top[tid]) : "memory");
    cluster_arrive();
    cluster_wait();
    if (part) return;
    t = sh.sums[0];
    for (int p = 1; p < parts; ++p) t = join(t, sh.sums[p], c);
    if (kTop) {
      __syncthreads();  // sh.top was read above
      rank_by_counting(sh.theirs, parts * a.top, a.top, sh.top);
      __syncthreads();
    }
  }
  const bool empty = t.s == 0.0f;  // the largest logit adds 1
  const float log_sum = logf(t.s);
  if (tid == 0) {
    float lp = 0.0f;
    if (target >= a.vocab) {
      flag_error(kErrCacheId);
      lp = NAN;
    } else if (target >= 0) {
      const float x = sizeof(T) == 2 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(row.x)[target] << 16)
                                     : reinterpret_cast<const float *>(row.x)[target];
      lp = empty ? -INFINITY : (x - t.m) * a.scale - log_sum;
    }
    a.logprob[i] = lp;
    if (a.entropy) a.entropy[i] = empty ? 0.0f : log_sum - 0.6931471805599453094f * t.h / t.s;
  }
  if (kTop && tid < a.top) {
    const uint64_t r = sh.top[tid];
    a.top_ids[(int64_t)i * a.top + tid] = index_in(r);
    a.top_logprobs[(int64_t)i * a.top + tid] = empty ? -INFINITY : (value_of(order_in(r)) - t.m) * a.scale - log_sum;
  }
}

template <typename T, bool kTop>
static cudaError_t launch(const LogprobArgs &a, cudaStream_t s) {
  // blocks for the whole GPU (152 SMs, 4 blocks each) from few rows, none with less than 4 KB
  const int64_t pieces = (int64_t)a.vocab / Piece<T>::kN + 2;
  int parts = 1;
  while (parts < kClusterMost && (int64_t)a.n * parts * 2 <= 152 * 4 && pieces / (parts * 2) >= 256) parts *= 2;
  int cell_log = 0;
  while ((pieces / parts + 1) >> cell_log >= kCells) ++cell_log;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)a.n * parts);
  cfg.blockDim = dim3(kThreads_);
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = parts;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, logprob_kernel<T, kTop>, a, parts, cell_log);
}

cudaError_t launch_token_logprobs(int dtype, const LogprobArgs &a, cudaStream_t s) {
  if (a.n == 0) return cudaSuccess;
  g_used = true;
  if (dtype == COPES_BF16) return a.top ? launch<__nv_bfloat16, true>(a, s) : launch<__nv_bfloat16, false>(a, s);
  return a.top ? launch<float, true>(a, s) : launch<float, false>(a, s);
}

unsigned read_and_clear_logprob_errors() {
  if (!g_used) return 0;
  unsigned v = 0, zero = 0;
  cudaMemcpyFromSymbol(&v, g_logprob_error, sizeof(v));
  if (v) cudaMemcpyToSymbol(g_logprob_error, &zero, sizeof(zero));
  return v;
}

}  // namespace copes
