// Log probabilities of given tokens, with entropy and top alternatives, from one pass over the
// logits.
//
// With m the row's maximum, y_j = scale (x_j - m) log2 e, s = sum 2^y_j and h = sum y_j 2^y_j:
//   logprob of t = scale (x_t - m) - ln s,   entropy = ln s - ln 2 h / s.
// A warp keeps a running m of what it has read and rescales its sums where that grows by
// g = scale (m' - m) log2 e (h' = 2^-g (h - g s)), so each logit is read once.  y is held at
// kLeast or above, where 2^y is 0: a masked token adds 0 to both sums.  A logit costs
// one exponential and about six more instructions, and HBM bounds it: 4,096 rows of 151,936 in bf16
// take 180 us, 6.9 TB/s (a plain copy: 6.8), and 215 us, 5.8 TB/s, with 20 alternatives: the ends
// of the rows, chains of loads and barriers, are partly hidden by the other blocks of an SM.
//
// The alternatives need no second pass over the row: while it is read, the maximum of every cell
// (a thread's pieces of one step, or of a few) is kept in shared memory, and each thread's over
// all in two halves.  The halves of one lane number are a group: the k-th largest of the 64 groups'
// maxima is a bound that k logits at least reach, so only cells that reach it hold alternatives.
// To fill k of 64 groups takes 64 (1/64 + ... + 1/(65 - k)) random logits, 24 for k = 20 and 44 for
// k = 32 (of 32 groups it would be 31 and 130): so many cells of thousands are read again, from L2,
// and their logits that reach the bound are ranked by counting.
//
// A row is read by one block, or, where rows alone would leave SMs without work, by a cluster of
// up to 8 blocks whose first joins the others' sums and alternatives through its shared memory.
#include <float.h>
#include <math.h>

#include "answer.h"

namespace copes {

__device__ unsigned g_logprob_error;
static std::atomic<bool> g_used{false};
__device__ __forceinline__ void flag_error(unsigned bit) { atomicOr(&g_logprob_error, bit); }

constexpr unsigned kAll = 0xffffffffu;
constexpr int kMostThreads = 256, kMostWarps = kMostThreads / 32;
// blocks of an SM: with a thread's next step on its way (shallow), or the next two (deep).  (With alternatives
// three of the four variants spill 4 or 8 bytes of a thread in the registers that this leaves.)
constexpr int per_sm(bool deep) { return deep ? 3 : 4; }
constexpr int kThreadCells = 48;   // of a thread, at most
constexpr int kReached = 512;      // cells read again by the fast way, at most
constexpr int kCandidates = 320;   // logits ranked by counting, at most
constexpr int kClusterMost = 8;
constexpr int kLoads = 4;          // 16-byte pieces of a lane in one step
// Shared memory of an SM that its blocks' cells may fill.  The rest of the 228 KB holds what loads
// have on their way: 1,216 rows of 151,936 with 20 alternatives take 67.5 us with 132 KB for the
// cells, 74.7 with 227, and 68.6 with 100, where cells of twice the size are read again.
constexpr int kShared = 132 << 10;
constexpr int kStep = kLoads * 32;  // pieces of a warp in one step

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
__device__ __forceinline__ float warp_max_nan(float x) {
  float r;
  asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
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

// A logit as it is kept in shared memory: in the logits' own bits.
template <typename T>
struct Kept {
  using Bits = uint32_t;
  __device__ static Bits from(float x) { return __float_as_uint(x); }
  __device__ static float to(Bits b) { return __uint_as_float(b); }
};
template <>
struct Kept<__nv_bfloat16> {
  using Bits = uint16_t;
  __device__ static Bits from(float x) { return (uint16_t)(__float_as_uint(x) >> 16); }
  __device__ static float to(Bits b) { return __uint_as_float((uint32_t)b << 16); }
};

template <typename T>
__device__ __forceinline__ Piece<T> load_piece(const void *at) {
  Piece<T> p;
  asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(p.r[0]), "=r"(p.r[1]), "=r"(p.r[2]), "=r"(p.r[3]) : "l"(at));
  return p;
}

// A row in aligned pieces of 16 bytes: piece v holds logits v kN - shift and on; the first and
// the last may hold fewer than kN.
template <typename T>
struct Row {
  const T *x;
  int vocab, shift;
  __device__ Row(const T *row, int n) : x(row), vocab(n), shift((int)(((uintptr_t)row & 15) / sizeof(T))) {}
  __device__ int pieces() const { return (int)(((int64_t)shift + vocab + Piece<T>::kN - 1) / Piece<T>::kN); }
  // pieces [first_full(), end_full()) are whole
  __device__ int first_full() const { return shift ? 1 : 0; }
  __device__ int end_full() const { return (int)(((int64_t)shift + vocab) / Piece<T>::kN); }
  __device__ const char *at(int v) const { return reinterpret_cast<const char *>(x - shift) + (int64_t)v * 16; }
  __device__ int first(int v) const { return v * Piece<T>::kN - shift; }
  // what lies outside the row reads as -inf
  __device__ __forceinline__ Piece<T> load(int v) const {
    Piece<T> p{};
    const int j = first(v);
    if (j >= 0 && j + Piece<T>::kN <= vocab) return load_piece<T>(x + j);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        p.r[i] = j + i >= 0 && j + i < vocab ? reinterpret_cast<const uint32_t *>(x)[j + i] : 0xFF800000u;
    } else {
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {  // few pieces of a row: short code
        uint32_t u = 0xFF80u, w = 0xFF80u;
        if (j + 2 * i >= 0 && j + 2 * i < vocab) u = reinterpret_cast<const uint16_t *>(x)[j + 2 * i];
        if (j + 2 * i + 1 >= 0 && j + 2 * i + 1 < vocab) w = reinterpret_cast<const uint16_t *>(x)[j + 2 * i + 1];
        p.r[0] = p.r[1];
        p.r[1] = p.r[2];
        p.r[2] = p.r[3];
        p.r[3] = u | w << 16;
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

// (Not .aligned: that asks for warps whose lanes are together, which after branches by lane nothing but the compiler sees to.)
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait;" ::: "memory"); }
// The address of the cluster's first block's copy of a shared variable.
__device__ __forceinline__ uint32_t in_first(const void *p) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)));
  return r;
}

// n <= 8 sums together, to the same bits in every lane.
__device__ __forceinline__ Sums warp_join(const Sums *from, int n, float c) {
  const int lane = threadIdx.x & 31;
  Sums t = lane < n ? from[lane] : Sums{-FLT_MAX, 0.0f, 0.0f};
  const float M = warp_max_nan(t.m);
  rebase(t.s, t.h, t.m, M, c);
#pragma unroll
  for (int d = 1; d < kMostWarps; d <<= 1) {
    t.s += __shfl_xor_sync(kAll, t.s, d);
    t.h += __shfl_xor_sync(kAll, t.h, d);
  }
  return {M, __shfl_sync(kAll, t.s, 0), __shfl_sync(kAll, t.h, 0)};
}
static_assert(kMostWarps <= 8 && kClusterMost <= 8, "warp_join adds up 8 lanes");

struct LogprobShared {
  union {
    alignas(16) uint64_t candidate[kCandidates];
    int group[2][kMostThreads];  // read before there are candidates
  };
  uint64_t top[COPES_MAX_TOP];
  uint16_t reached[kReached];  // cells that reach the bound
  Sums sums[kClusterMost];
  int bound;
  Sums warp[kMostWarps];
  uint64_t best[kMostWarps];
  int n_reached, n_candidates;
};

// top[0 .. k): the k largest of list[0 .. n), untouched past them.  By counting: the numbers differ.
__device__ __forceinline__ void rank_by_counting(const uint64_t *list, int n, int k, uint64_t *top) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const uint64_t mine = list[i];
    int rank = n & 1 ? list[n - 1] > mine : 0;
#pragma unroll 8
    for (int j = 0; j < n / 2; ++j) {
      const ulonglong2 two = reinterpret_cast<const ulonglong2 *>(list)[j];
      rank += (two.x > mine) + (two.y > mine);
    }
    if (rank < k && mine) top[rank] = mine;
  }
}

// A place for `mine` entries of each lane in a list of which *n are taken.
__device__ __forceinline__ int warp_reserve(int mine, int *n) {
  if (!__any_sync(kAll, mine)) return 0;
  const int lane = threadIdx.x & 31;
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(kAll, upto, d);
    if (lane >= d) upto += y;
  }
  int at = 0;
  if (lane == 31) at = atomicAdd(n, upto);
  return __shfl_sync(kAll, at, 31) + upto - mine;
}

// visit(a logit's order, its index) for the logits of piece v whose order is `least` or above.
template <typename T, typename Visit>
__device__ __forceinline__ void visit_piece(const Row<T> &row, int v, int least, Visit visit) {
  constexpr int N = Piece<T>::kN;
  const Piece<T> p = row.load(v);
  if (order_of(max_of(p)) < least) return;
  const int j = row.first(v);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    float x[2];
    pair_of(p, e / 2, x[0], x[1]);
    const int o = order_of(x[e & 1]);
    if (o >= least && (unsigned)(j + e) < (unsigned)row.vocab) visit(o, (uint32_t)(j + e));
  }
}

// The k largest of pieces [v0, v0 + n) where the logits that reach the bound are too many to be
// listed.  Where most of them equal it (masked tokens, with fewer than k others): those that surpass
// it and, in the order of the indices, the first that equal it.  Else one after the other.
template <typename T>
__device__ __noinline__ void find_top_slowly(LogprobShared &sh, const typename Kept<T>::Bits *cell, const Row<T> &row, int v0, int n,
                                             int merge, int bound, int k) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  // visits the thread's own logits of order `least` and above, by its cells' maxima
  const auto each = [&](int least, auto visit) {
    const int steps = (n + kStep * warps - 1) / (kStep * warps);
    for (int step = 0; step < steps; ++step) {
      if (order_of(Kept<T>::to(cell[(step >> merge) * blockDim.x + tid])) < least) continue;
      for (int u = 0; u < kLoads; ++u) {
        const int v = ((step * warps + warp) * kLoads + u) * 32 + lane;
        if (v < n) visit_piece(row, v0 + v, least, visit);
      }
    }
  };
  __syncthreads();
  if (tid == 0) sh.n_candidates = 0;
  __syncthreads();
  if (bound != 0x7FFFFFFF)
    each(bound + 1, [&](int order, uint32_t index) {
      const int at = atomicAdd(&sh.n_candidates, 1);
      if (at < kCandidates) sh.candidate[at] = ranked(order, index);
    });
  __syncthreads();
  const int above = sh.n_candidates;
  if (above <= kCandidates - COPES_MAX_TOP) {
    if (warp == 0) {
      int equal = 0;
      for (int v = lane; equal < k && v - lane < n; v += 32) {
        int mine = 0;
        if (v < n) visit_piece(row, v0 + v, bound, [&](int order, uint32_t) { mine += order == bound; });
        int before = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int y = __shfl_up_sync(kAll, before, d);
          if (lane >= d) before += y;
        }
        int at = equal + before - mine;
        equal += __shfl_sync(kAll, before, 31);
        if (mine && at < k)
          visit_piece(row, v0 + v, bound, [&](int order, uint32_t index) {
            if (order == bound && at < k) sh.candidate[above + at++] = ranked(bound, index);
          });
      }
      if (lane == 0) sh.n_candidates = above + min(equal, k);
    }
    __syncthreads();
    rank_by_counting(sh.candidate, sh.n_candidates, k, sh.top);
    __syncthreads();
    return;
  }
  uint64_t last = ~0ull;
  for (int r = 0; r < k; ++r) {
    uint64_t next = 0;
    each(bound, [&](int order, uint32_t index) {
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
    for (int w = 0; w < warps; ++w)
      if (sh.best[w] > next) next = sh.best[w];
    if (tid == 0) sh.top[r] = next;
    last = next;
    __syncthreads();
  }
}

// The k-th largest (1 <= k <= 32) of a warp's 64 numbers: a bitonic sort, the largest in a of lane 0.
__device__ __forceinline__ int kth_of_64(int a, int b, int k) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int d = size >> 1; d; d >>= 1) {
      const int u = __shfl_xor_sync(kAll, a, d), v = __shfl_xor_sync(kAll, b, d);
      const bool lower = (lane & d) == 0;
      const bool down = size == 32 || (lane & size) == 0;  // a's second halves and, last, all of b ascend
      a = down == lower ? max(a, u) : min(a, u);
      b = (size == 32 ? false : down) == lower ? max(b, v) : min(b, v);
    }
  int top = max(a, b);  // the 32 largest, in some order
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const int u = __shfl_xor_sync(kAll, top, d);
    top = (lane & d) == 0 ? max(top, u) : min(top, u);
  }
  return __shfl_sync(kAll, top, k - 1);
}

// The block's alternatives into sh.top, from the cells' maxima of pieces [v0, v0 + n) and `own`,
// this thread's over all, in two halves.  cell[j blockDim + tid]: steps j 2^merge and on of the thread.
template <typename T>
__device__ __forceinline__ void find_top(LogprobShared &sh, const typename Kept<T>::Bits *cell, const Row<T> &row, int v0, int n, int merge,
                                         const float (&own)[2], int k) {
  constexpr int N = Piece<T>::kN;
  const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x, warps = threads >> 5;
  sh.group[0][tid] = order_of(own[0]);
  sh.group[1][tid] = order_of(own[1]);
  __syncthreads();
  if (tid < 32) {
    int u = sh.group[0][lane], v = sh.group[1][lane];
    for (int w = 1; w < warps; ++w) {
      u = max(u, sh.group[0][w * 32 + lane]);
      v = max(v, sh.group[1][w * 32 + lane]);
    }
    u = kth_of_64(u, v, k);
    if (lane == 0) sh.bound = u;
  }
  __syncthreads();
  const int bound = sh.bound;
  {
    uint64_t mine = 0;  // which of the thread's cells, at most kThreadCells
    if (order_of(max_nan(own[0], own[1])) >= bound) {
      const int steps = (n + kStep * warps - 1) / (kStep * warps), cells = (steps + (1 << merge) - 1) >> merge;
#pragma unroll 4
      for (int j = 0; j < cells; ++j) mine |= (uint64_t)(order_of(Kept<T>::to(cell[j * threads + tid])) >= bound) << j;
    }
    int at = warp_reserve(__popcll(mine), &sh.n_reached);
    for (; mine; mine &= mine - 1, ++at)
      if (at < kReached) sh.reached[at] = (uint16_t)((__ffsll(mine) - 1) * threads + tid);
  }
  __syncthreads();
  const int reached = sh.n_reached;
  bool listed = reached <= kReached;
  if (listed) {
    const int sub = 2 + merge, shift = 31 - __clz(threads), items = reached << sub;  // 2^sub pieces in a cell
    for (int base = tid & ~31; base < items; base += threads) {
      const int i = base + lane;
      Piece<T> p;
      int j = 0, mine = 0;
      if (i < items) {
        const int id = sh.reached[i >> sub], part = i & ((1 << sub) - 1);
        const int step = ((id >> shift) << merge) + (part >> 2), thread = id & (threads - 1);
        const int v = ((step * warps + (thread >> 5)) * kLoads + (part & 3)) * 32 + (thread & 31);
        if (v < n) {
          p = row.load(v0 + v);
          j = row.first(v0 + v);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            float x[2];
            pair_of(p, e / 2, x[0], x[1]);
            mine |= (order_of(x[e & 1]) >= bound && (unsigned)(j + e) < (unsigned)row.vocab) << e;
          }
        }
      }
      int at = warp_reserve(__popc(mine), &sh.n_candidates);
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (mine >> e & 1) {
          float x[2];
          pair_of(p, e / 2, x[0], x[1]);
          if (at < kCandidates) sh.candidate[at] = ranked(order_of(x[e & 1]), (uint32_t)(j + e));
          ++at;
        }
    }
    __syncthreads();
    const int found = sh.n_candidates;
    listed = found <= kCandidates;
    if (listed) {
      rank_by_counting(sh.candidate, found, k, sh.top);
      __syncthreads();
    }
  }
  if (!listed) find_top_slowly(sh, cell, row, v0, n, merge, bound, k);
}

// A block, or a cluster of `parts` blocks, per row; a cell is 2^merge steps of a thread.  Before it
// looks for a row's alternatives a block asks for the first kAhead bytes (a quarter at most) of what a
// block `apart` rows on reads, whose turn is near, into L2, so that HBM is not idle meanwhile.
constexpr int kAhead = 48 << 10;

template <typename T, bool kTop, bool kDeep>
__global__ void __launch_bounds__(kMostThreads, per_sm(kDeep)) logprob_kernel(LogprobArgs a, int parts, int merge, int apart, int cell_bytes) {
  extern __shared__ __align__(16) unsigned char dynamic[];
  auto *const cell = reinterpret_cast<typename Kept<T>::Bits *>(dynamic);
  __shared__ LogprobShared sh;
  constexpr int N = Piece<T>::kN;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5, stride = warps * kStep;
  const int part = blockIdx.x % parts;
  const int64_t i = blockIdx.x / parts;
  // launched while the kernel before it on the stream ends, whose results are waited for here
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float c = a.scale * 1.44269504088896340736f;
  const uint64_t c2 = pack2(c, c);
  if (parts > 1) cluster_arrive();
  const Row<T> row((const T *)a.logits + i * a.row, a.vocab);
  const int all = row.pieces();
  const int v0 = (int)((int64_t)all * part / parts), n = (int)((int64_t)all * (part + 1) / parts) - v0;
  const int full0 = row.first_full() - v0, full1 = min(n, row.end_full() - v0);
  const char *at = row.at(v0) + lane * 16;
  const int64_t target = a.target[i];

  Sums t{-FLT_MAX, 0.0f, 0.0f};
  float own[2] = {-INFINITY, -INFINITY};
  uint64_t s2 = 0, h2 = 0;
  Piece<T> now[kLoads], next[kLoads], then[kLoads];
  const auto fetch = [&](int base, Piece<T>(&to)[kLoads]) {
    if (base >= full0 && base + kStep <= full1) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) to[u] = load_piece<T>(at + (int64_t)base * 16 + u * 512);
      return;
    }
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
  if constexpr (kDeep)
    if (warp * kStep + stride < n) fetch(warp * kStep + stride, next);
  if (kTop) {
    if (tid < COPES_MAX_TOP) sh.top[tid] = 0;
    if (tid == 0) sh.n_reached = sh.n_candidates = 0;
  }
  int step = 0;
  const auto take = [&](const Piece<T>(&p)[kLoads]) {
    const float half[2] = {max_nan(max_of(p[0]), max_of(p[1])), max_nan(max_of(p[2]), max_of(p[3]))};
    const float most = max_nan(half[0], half[1]);
    if (kTop) {
      own[0] = max_nan(own[0], half[0]);
      own[1] = max_nan(own[1], half[1]);
      auto *to = cell + (step >> merge) * blockDim.x + tid;
      *to = Kept<T>::from(step & ((1 << merge) - 1) ? max_nan(Kept<T>::to(*to), most) : most);
    }
    const float M = max_nan(t.m, warp_max_nan(most));
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
        pair_of(p[u], e, x, y);
        unpack2(mul2(add2(pack2(x, y), minus_m), c2), x, y);
        x = max_nan(x, kLeast);
        y = max_nan(y, kLeast);
        const uint64_t q = pack2(exp2_fast(x), exp2_fast(y));
        s2 = add2(s2, q);
        h2 = fma2(q, pack2(x, y), h2);
      }
    ++step;
  };
  // The buffers take turns (4,096 rows: 180 us, where each moves on 188; 1,216 with 20 alternatives 69
  // and 73; 2,000 rows of fp32 with 20 190 and 203).  Of bf16 with two steps ahead and alternatives
  // each moves on: three copies of that loop, of twice the logits, beside the end of a row are too
  // much code (225 us in turns, 215 so).
  for (int base = warp * kStep; base < n;) {
    const auto turn = [&](const Piece<T>(&p)[kLoads], Piece<T>(&later)[kLoads]) {
      if (base + (kDeep ? 2 : 1) * stride < n) fetch(base + (kDeep ? 2 : 1) * stride, later);
      take(p);
      base += stride;
      return base < n;
    };
    if constexpr (kDeep && kTop && sizeof(T) == 2) {
      if (!turn(now, then)) break;
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        now[u] = next[u];
        next[u] = then[u];
      }
    } else if constexpr (kDeep) {
      if (!turn(now, then) || !turn(next, now)) break;
      turn(then, next);
    } else {
      if (!turn(now, next)) break;
      turn(next, now);
    }
  }
  if (tid == 0 && i + apart < a.n) {
    const Row<T> later((const T *)a.logits + (i + apart) * a.row, a.vocab);
    const int v = max((int)((int64_t)later.pieces() * part / parts), later.first_full());
    const int bytes = min(min(n, later.end_full() - v), min(kAhead / 16, n / 4)) * 16;
    if (bytes > 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(later.at(v)), "r"(bytes) : "memory");
  }
  if (kTop) {  // a thread's steps past its last hold nothing
    const int steps = (n + stride - 1) / stride, cells = (steps + (1 << merge) - 1) >> merge;
    for (int j = (step + (1 << merge) - 1) >> merge; j < cells; ++j) cell[j * blockDim.x + tid] = Kept<T>::from(-INFINITY);
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
  t = warp_join(sh.warp, warps, c);
  if (kTop) find_top(sh, cell, row, v0, n, merge, own, a.top);

  if (parts > 1) {
    uint64_t *const theirs = reinterpret_cast<uint64_t *>(dynamic + cell_bytes);  // of the cluster's blocks, in the first
    cluster_wait();  // the first block has begun
    const uint32_t to = in_first(&sh.sums[part]);
    if (tid < 3)
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4 * tid), "f"(tid == 0 ? t.m : tid == 1 ? t.s : t.h)
                   : "memory");
    if (kTop && tid < a.top)
      asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(in_first(theirs + part * a.top + tid)), "l"(sh.top[tid])
                   : "memory");
    cluster_arrive();
    cluster_wait();
    if (part) return;
    t = warp_join(sh.sums, parts, c);
    if (kTop) {
      rank_by_counting(theirs, parts * a.top, a.top, sh.top);  // sh.top was read before the barrier
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
    a.top_ids[i * a.top + tid] = index_in(r);
    a.top_logprobs[i * a.top + tid] = empty ? -INFINITY : (value_of(order_in(r)) - t.m) * a.scale - log_sum;
  }
}

// How a call is cut: blocks of a row, threads of a block, 2^merge steps that share a cell, blocks the
// GPU runs at once, one step ahead or two.
struct Cut {
  int parts, threads, merge, at_once;
  bool deep;
  uint32_t cell_bytes;
};

// The cut that costs least by this count: waves of blocks over the GPU, times the blocks that run at
// once (a block's share of HBM), times a block's pieces and what its beginning and end cost it,
// 24 pieces' time a thread with alternatives and 16 without.  A block has a step for each thread at
// least, and 256 pieces where it is one of several of a row; with one step ahead instead of two a
// long row takes 5% longer, 15% with 64 threads.  One warp alone is for rows too short for two: the
// end of a row is a chain of loads that more warps shorten.  What it decides, in us with 5 alternatives (bf16 where nothing is said):
//   rows x logits     parts 1, 2, 4, 8             threads 32, 64, 128, 256 (two steps ahead)
//   38 x 151,936      15.1, 12.1, 10.7, 10.3
//   120 x 151,936     18.4, 15.8, 20.6, 26.1
//   300 x 151,936     23.5, 32.1, 35.2, 53.2
//   4,096 x 151,936                                -, -, 211, 220
//   4,096 x 32,003                                 68, 60, 65, 84
//   20,000 x 32,003                                296, 252, 292, 396
//   500 x 7,500                                    9.3, 8.0, 7.4, 7.6
// and steps ahead, 500 x 151,936 (one wave or two): 38 with one, 45 with two; 734 x 151,936: 58, 47.
static Cut cut_of(int64_t n, int64_t pieces, bool top, int size) {
  Cut best{1, 32, 0, 152, false, 0};
  double least = 0.0;
  for (int parts = 1; parts <= kClusterMost && (parts == 1 || pieces / parts >= 256); parts *= 2) {
    const int64_t mine = pieces / parts + 1;
    for (int threads = mine >= 64 * kLoads ? 64 : 32; threads <= kMostThreads && (threads <= 64 || mine >= threads * kLoads);
         threads *= 2)
      for (int deep = 0; deep < 2; ++deep) {
        const int64_t at_once = (int64_t)152 * per_sm(deep) * (kMostThreads / threads);
        const bool longer = mine >= 3 * threads * kLoads;
        if (deep && !longer) continue;
        const int64_t waves = (n * parts + at_once - 1) / at_once;
        const double cost = (double)(waves * at_once) * (double)(mine + (top ? 24 : 16) * threads) *
                            (deep || !longer ? 1.0 : threads <= 64 ? 1.15 : 1.05);
        if (least == 0.0 || cost < least) {
          least = cost;
          best = Cut{parts, threads, 0, (int)at_once, deep != 0, 0};
        }
      }
  }
  const int64_t mine = pieces / best.parts + 1, steps = (mine + best.threads * kLoads - 1) / (best.threads * kLoads);
  const int64_t room = kShared / (best.at_once / 152) - 1024 - (int64_t)sizeof(LogprobShared);
  // few cells are not worth merging: what they save is less than an SM has
  const auto cells = [&] { return (steps + (1 << best.merge) - 1) >> best.merge; };
  while (cells() > kThreadCells || (cells() > 8 && cells() * best.threads * size > room)) ++best.merge;
  best.cell_bytes = top ? (uint32_t)cells() * best.threads * size : 0;
  return best;
}

template <typename T, bool kTop, bool kDeep>
static cudaError_t launch(const LogprobArgs &a, const Cut &c, cudaStream_t s) {
  const auto kernel = logprob_kernel<T, kTop, kDeep>;
  const uint32_t bytes = c.cell_bytes + (kTop && c.parts > 1 ? c.parts * a.top * 8 : 0), fixed = sizeof(LogprobShared);
  const cudaError_t e = allow_smem((const void *)kernel, bytes + fixed, kThreadCells * kMostThreads * 4 + kClusterMost * COPES_MAX_TOP * 8);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)a.n * c.parts);
  cfg.blockDim = dim3(c.threads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = c.parts;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = c.parts > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, c.parts, c.merge, c.at_once / c.parts, (int)c.cell_bytes);
}

template <typename T, bool kTop>
static cudaError_t launch_any(const LogprobArgs &a, cudaStream_t s) {
  const Cut c = cut_of(a.n, (int64_t)a.vocab / Piece<T>::kN + 2, kTop, sizeof(T));
  return c.deep ? launch<T, kTop, true>(a, c, s) : launch<T, kTop, false>(a, c, s);
}

cudaError_t launch_token_logprobs(int dtype, const LogprobArgs &a, cudaStream_t s) {
  if (a.n == 0) return cudaSuccess;
  g_used = true;
  if (dtype == COPES_BF16) return a.top ? launch_any<__nv_bfloat16, true>(a, s) : launch_any<__nv_bfloat16, false>(a, s);
  return a.top ? launch_any<float, true>(a, s) : launch_any<float, false>(a, s);
}

unsigned read_and_clear_logprob_errors() {
  if (!g_used) return 0;
  unsigned v = 0, zero = 0;
  cudaMemcpyFromSymbol(&v, g_logprob_error, sizeof(v));
  if (v) cudaMemcpyToSymbol(g_logprob_error, &zero, sizeof(zero));
  return v;
}

}  // namespace copes
