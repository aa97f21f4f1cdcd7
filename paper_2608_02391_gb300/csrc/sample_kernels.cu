// The next token of each row of logits from a given random number, with the usual cuts.
//
// Every token has a weight that is a whole number, so that sums are exact in any order and a row's token
// does not depend on how the row was shared out: with m the row's largest logit,
//   t = (m - x) * (scale log2 e),  n = floor(t),  f = t - n   (each step rounded to fp32),
//   weight = floor(P(f) 2^(40 - n)),   P(f) = 2^-f within 2^-21 (Horner's steps fused; power below).
// The tokens in order of falling logit, equal ones by ascending id, are cut to the first top_k, to the
// shortest beginning that holds top_p of their weight, and to t <= -log2 min_p.  Of the tokens kept, in
// ascending id, the one drawn is the first at which the sum of the weights passes
// floor(floor(u 2^31) total / 2^31).
//
// A row is read by a block, or by a cluster of up to 8 where rows alone would leave SMs without work: from HBM
// for its maximum, and then from L2 for what follows.  A weight takes 13 operations of the fp32 units, by
// pairs, and 5 others, so a pass over 151,936 of them keeps an SM for 14 us, where HBM brings that row in bf16 in 7:
// 2,048 rows without a cut take 236 us, 190 of them these passes, in which one of an SM's two blocks computes while the
// other reads (to have the next row brought to L2 by the pass over this one, or its maximum found by it, or the second
// blocks begin later, made nothing faster).
//
// Cuts.  While the maximum is sought, each thread keeps the maxima of four cells of the row: the k-th
// largest of the 2,048 cells is a bound that k logits at least reach.  Those that do (a few more than k, as a
// rule; 128 for a top_p alone) are collected, cut and drawn from, in shared memory: 608 rows take 57 us with top_k
// 50, 98 with top_p 0.95 where few tokens hold that.  A cut that lies behind them (of a flat row) is sought by a
// count of tokens by their distance: the tokens near it are collected, what is nearer is summed exactly, and
// the token drawn from the sums of chunks: 253 us.  Where thousands of logits are equal, passes bracket the cut.
#include <float.h>
#include <math.h>

#include "answer.h"
#include "copes_device.cuh"

namespace copes {

__device__ unsigned g_sample_error;
static std::atomic<bool> g_used{false};
__device__ __forceinline__ void flag_error(unsigned bit) { atomicOr(&g_sample_error, bit); }

namespace {

constexpr unsigned kAll = 0xffffffffu;
constexpr int kEach = 4;                   // pieces of 16 bytes of a lane in a chunk, and cells of a thread
constexpr int kChunkPieces = 32 * kEach;
constexpr int kList = 2048;                // logits that can be collected
constexpr int kMaxCluster = 8;
constexpr float kFarthest = 40.0f;         // the weight is 0 past it
constexpr int kBinsOfOne = 64, kBins = 40 * kBinsOfOne + 1;
using u64 = unsigned long long;

// P(f) = 1 + f Q(f): Q of degree 4 that makes the largest |P 2^f - 1| on [0, 1] least (1.6e-7 before rounding),
// with P at most 1 and at least 1/2.
__device__ __forceinline__ float power(float f) {
  float p = -0.0008996404358185828f;
  p = fmaf(p, f, 0.009098555892705917f);
  p = fmaf(p, f, -0.05521015450358391f);
  p = fmaf(p, f, 0.2401522845029831f);
  p = fmaf(p, f, -0.693140983581543f);
  return fmaf(p, f, 1.0f);
}

// The weight of a token at distance t: P lies in [1/2, 1], so its bits less those of 1/4 are P 2^24.
__device__ __forceinline__ u64 weight_of(float t) {
  t = fminf(t, 63.0f);
  const float z = __fadd_rd(t, 8388608.0f);  // 2^23 + n
  const uint32_t p = __float_as_uint(power(t - (z - 8388608.0f))) - 0x3E800000u;
  return ((u64)p << 16) >> (__float_as_uint(z) & 63u);
}

// Two floats in a register pair (pack_f32x2), added downwards and upwards.
using Pair = u64;
__device__ __forceinline__ float2 floats_of(Pair p) {
  float2 f;
  unpack_f32x2(p, f.x, f.y);
  return f;
}
__device__ __forceinline__ Pair add2_down(Pair a, Pair b) {
  Pair d;
  asm("add.rm.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ Pair add2_up(Pair a, Pair b) {
  Pair d;
  asm("add.rp.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// -t of two tokens: (x - m) c, each operation rounded.
__device__ __forceinline__ Pair minus_t(float x0, float x1, float m, float c) {
  return mul_f32x2(add_f32x2(pack_f32x2(x0, x1), splat_f32x2(-m)), splat_f32x2(c));
}

// The sum of the weights of at most 60 tokens, and their number, in 32-bit registers.  With y = P(f) 2^-n, whose
// bits are P's less n in the exponent, a weight is floor(y 2^40): 2^23 floor(y 2^17), which is what adding 64
// downwards leaves in the last bits, and floor(rest 2^40), by 2^-17 likewise (2^-17 less the upper part is exact).
// The upper 9 bits of 64's, 133 each, count the tokens.  (With 64-bit shifts and additions, and each token for itself,
// 2,048 rows of 151,936 took 377 us; with the upper part taken from y first, and then 2^-17 added, 250.)
struct Weights {
  uint32_t hi = 0, lo = 0;
  // Tokens at -minus.x and -minus.y, where keep.
  __device__ __forceinline__ void add(Pair minus, bool keep_x, bool keep_y) {
    const Pair z = add2_up(minus, splat_f32x2(12582912.0f));  // 1.5 2^23 - n
    const Pair less = add_f32x2(z, splat_f32x2(-12582912.0f));  // -n
    const Pair f = fma_f32x2(minus, splat_f32x2(-1.0f), less);
    Pair p = splat_f32x2(-0.0008996404358185828f);
    p = fma_f32x2(p, f, splat_f32x2(0.009098555892705917f));
    p = fma_f32x2(p, f, splat_f32x2(-0.05521015450358391f));
    p = fma_f32x2(p, f, splat_f32x2(0.2401522845029831f));
    p = fma_f32x2(p, f, splat_f32x2(-0.693140983581543f));
    p = fma_f32x2(p, f, splat_f32x2(1.0f));
    const float2 zz = floats_of(z), pp = floats_of(p);
    const Pair y = pack_f32x2(__uint_as_float(__float_as_uint(pp.x) + (__float_as_uint(zz.x) << 23)),
                              __uint_as_float(__float_as_uint(pp.y) + (__float_as_uint(zz.y) << 23)));
    const Pair top = add2_down(y, splat_f32x2(64.0f));
    const Pair rest = add2_down(fma_f32x2(top, splat_f32x2(-1.0f), splat_f32x2(64.0f + 0x1p-17f)), y);
    const float2 t = floats_of(top), r = floats_of(rest);
    if (keep_x) {
      hi += __float_as_uint(t.x);
      lo += __float_as_uint(r.x);
    }
    if (keep_y) {
      hi += __float_as_uint(t.y);
      lo += __float_as_uint(r.y);
    }
  }
  __device__ __forceinline__ uint32_t tokens() const { return (hi >> 23) * 77u & 511u; }  // 77 * 133 = 1 (mod 512)
  __device__ __forceinline__ u64 sum() const { return ((u64)(hi & 0x7FFFFFu) << 23) + (lo - tokens() * 0x37000000u); }
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float c;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(a), "f"(b));
  return c;
}

// A row in pieces of 16 aligned bytes; what lies outside the row is -infinity.
template <typename T>
struct Row {
  static constexpr int kN = 16 / (int)sizeof(T);
  const uint4 *base;
  const T *first;
  int shift, vocab, pieces;  // elements of the first piece before the row
  __device__ Row(const void *logits, int64_t row, int64_t i, int n) : first((const T *)logits + i * row), vocab(n) {
    shift = (int)(((uintptr_t)first & 15) / sizeof(T));
    base = reinterpret_cast<const uint4 *>((uintptr_t)first & ~(uintptr_t)15);
    pieces = (shift + n - 1) / kN + 1;
  }
  __device__ __forceinline__ int id(int piece) const { return piece * kN - shift; }
  __device__ __forceinline__ uint4 load(int piece) const {
    const int at = id(piece);
    if (at >= 0 && at + kN <= vocab) return base[piece];
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
#pragma unroll
    for (int e = 0; e < kN; ++e) {
      if (at + e < 0 || at + e >= vocab) continue;
      if constexpr (sizeof(T) == 4) {
        w[e] = reinterpret_cast<const uint32_t *>(first)[at + e];
      } else {
        const uint32_t x = reinterpret_cast<const uint16_t *>(first)[at + e];
        w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | x << 16 : (w[e / 2] & 0xFFFF0000u) | x;
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ static float element(const uint4 &p, int e) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
  __device__ __forceinline__ float at(int id) const {
    if constexpr (sizeof(T) == 4) return first[id];
    else return __bfloat162float(first[id]);
  }
  // An order of the elements (but NaN) as whole numbers of the type's size, +0 and -0 the same, and back.
  static constexpr int kBits = 8 * (int)sizeof(T);
  static constexpr uint32_t kInfinity = sizeof(T) == 4 ? 0xFF800000u : 0xFF80u, kNothing = sizeof(T) == 4 ? 0x007FFFFFu : 0x7Fu;
  __device__ __forceinline__ static uint32_t key(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return (u ^ (uint32_t)((int32_t)u >> 31 | 0x80000000)) >> (32 - kBits);
  }
  __device__ __forceinline__ static float value_of(uint32_t key) {
    const uint32_t u = key << (32 - kBits);
    return __uint_as_float(u >> 31 ? u ^ 0x80000000u : ~u & ~((1ull << (32 - kBits)) - 1));
  }
  // The largest element of a piece and of what `before` holds (as `none` at first), in the elements' own type.
  static constexpr uint32_t none = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
  __device__ __forceinline__ static uint32_t largest(uint32_t before, const uint4 &p) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) before = __float_as_uint(max_nan(__uint_as_float(before), __uint_as_float(w[e])));
      else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(before) : "r"(before), "r"(w[e]));
    }
    return before;
  }
  // Bits of a piece's elements in [low, high], those of its pieces j = 0 .. kEach - 1 apart, and a bit's j kN + e.
  __device__ __forceinline__ static uint32_t within(const uint4 &p, int j, float low, float high) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
    uint32_t found = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) {
        const float x = __uint_as_float(w[e]);
        if (x >= low && x <= high) found |= 1u << (4 * j + e);
      } else {
        const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&w[e]);
        found |= __hge2_mask(x, __float2bfloat162_rn(low)) & __hle2_mask(x, __float2bfloat162_rn(high)) & 0x10001u << (4 * j + e);
      }
    }
    return found;
  }
  __device__ __forceinline__ static int place(int bit) { return sizeof(T) == 4 ? bit : (bit & 15) * 2 + (bit >> 4); }
  __device__ __forceinline__ static float value(uint32_t largest) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(largest);
    else return max_nan(__uint_as_float(largest << 16), __uint_as_float(largest & 0xFFFF0000u));
  }
};

// What is in shared memory beside the list.
struct Shared {
  u64 sums[2][32][4];            // of warps, by turns
  u64 peers[2][kMaxCluster][4];  // of the blocks of a cluster
  u64 items[2][32][3];
  u64 scan[32];
  uint32_t counts[2][32];
  int collected;
  uint32_t first;  // upper half of the list's first entry
  u64 total;
  u64 held;  // the list's weight, where it is not all that was sought
  int chunk;
  int bins[2];  // first and last
};

__device__ __forceinline__ uint32_t remote(uint32_t at, int rank) {
  uint32_t to;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(at), "r"(rank));
  return to;
}

// The blocks that share a row: one, or a cluster.
template <int kWarps_>
struct Group {
  static constexpr int kWarps = kWarps_;
  static_assert((kWarps & (kWarps - 1)) == 0 && kWarps <= 32, "sums over warps by halves");
  int size, rank, turn;
  Shared *s;
  __device__ __forceinline__ void sync() const {
    if (size == 1) {
      __syncthreads();
    } else {
      // (not .aligned: lanes come here from branches of their own, and need not be together)
      asm volatile("barrier.cluster.arrive.release;" ::: "memory");
      asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
  }
  // v[j] over all threads, by adding or, kMax, as the largest; the same in every thread.
  template <int kM, bool kMax = false>
  __device__ __forceinline__ void all(u64 (&v)[kM]) {
    const auto join = [](u64 a, u64 b) { return kMax ? (a > b ? a : b) : a + b; };
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    turn ^= 1;
#pragma unroll
    for (int j = 0; j < kM; ++j) {
#pragma unroll
      for (int d = 16; d; d >>= 1) v[j] = join(v[j], __shfl_xor_sync(kAll, v[j], d));
      if (lane == 0) s->sums[turn][warp][j] = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kM; ++j) {
      v[j] = s->sums[turn][lane % kWarps][j];
#pragma unroll
      for (int d = kWarps / 2; d; d >>= 1) v[j] = join(v[j], __shfl_xor_sync(kAll, v[j], d));
    }
    if (size == 1) return;
    if (warp == 0 && lane < size)
#pragma unroll
      for (int j = 0; j < kM; ++j)
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(remote(smem_addr(&s->peers[turn][rank][j]), lane)), "l"(v[j]) : "memory");
    sync();
#pragma unroll
    for (int j = 0; j < kM; ++j) {
      v[j] = s->peers[turn][0][j];
      for (int r = 1; r < size; ++r) v[j] = join(v[j], s->peers[turn][r][j]);
    }
  }
};

// Runs f(chunk, its pieces of this lane) over this block's share of the row: chunk c is its where c % size ==
// rank, and a warp's as a whole.
template <typename T, int kWarps, typename F>
__device__ __forceinline__ void for_row(const Row<T> &row, const Group<kWarps> &g, const F &f) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int chunks = (row.pieces - 1) / kChunkPieces + 1;
  for (int c = g.rank + g.size * warp; c < chunks; c += g.size * kWarps) {
    uint4 p[kEach];
    const int first = c * kChunkPieces + lane;
    if (row.id(c * kChunkPieces) >= 0 && row.id((c + 1) * kChunkPieces) <= row.vocab) {
#pragma unroll
      for (int j = 0; j < kEach; ++j) p[j] = row.base[first + j * 32];
    } else {
#pragma unroll
      for (int j = 0; j < kEach; ++j) p[j] = row.load(first + j * 32);
    }
    f(c, p);
  }
}
// f(element, its id) for all of a lane's.
template <typename T, typename F>
__device__ __forceinline__ void for_chunk(const Row<T> &row, int chunk, const uint4 (&p)[kEach], const F &f) {
#pragma unroll
  for (int j = 0; j < kEach; ++j)
#pragma unroll
    for (int e = 0; e < Row<T>::kN; ++e)
      f(Row<T>::element(p[j], e), row.id(chunk * kChunkPieces + j * 32 + (int)(threadIdx.x & 31)) + e);
}

// Exclusive sums of v over the block's threads, and the total.
template <int kWarps>
__device__ __forceinline__ u64 block_scan(u64 v, Shared *s, u64 *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u64 x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u64 y = __shfl_up_sync(kAll, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // scan may still be read
  if (lane == 31) s->scan[warp] = x;
  __syncthreads();
  u64 before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += s->scan[w];
    sum += s->scan[w];
  }
  *total = sum;
  return before + x - v;
}

// Sums of v < 2^50 over a warp.
__device__ __forceinline__ u64 warp_sum(u64 v) {
  const uint32_t a = __reduce_add_sync(kAll, (uint32_t)v & 0x1FFFFFFu), b = __reduce_add_sync(kAll, (uint32_t)(v >> 25));
  return a + ((u64)b << 25);
}

// Collected tokens in the block's registers, kEvery of them in each thread's: entries, which ascend in
// the order of the tokens (keys falling, then ids rising), and weights.  Everything about them is found by
// searching for an answer two bits at a time, by three sums over the block, which sorts nothing.
template <int kEvery_, int kThreads>
struct Items {
  static constexpr int kEvery = kEvery_, kWarps = kThreads / 32;
  u64 entry[kEvery], weight[kEvery];
  int count, turn = 0;
  Shared *s;

  template <typename F>
  __device__ Items(const u64 *list, int n, Shared *shared, const F &weight_at) : count(n), s(shared) {
#pragma unroll
    for (int i = 0; i < kEvery; ++i) {
      const int at = i * kThreads + (int)threadIdx.x;
      entry[i] = at < n ? list[at] : ~0ull;
      weight[i] = at < n ? weight_at(list[at]) : 0;
    }
  }
  template <int kM>
  __device__ __forceinline__ void sums(u64 (&v)[kM]) {
#pragma unroll
    for (int j = 0; j < kM; ++j) v[j] = warp_sum(v[j]);
    const int lane = threadIdx.x & 31;
    turn ^= 1;
#pragma unroll
    for (int j = 0; j < kM; ++j)
      if (lane == 0) s->items[turn][threadIdx.x >> 5][j] = v[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kM; ++j) v[j] = warp_sum(lane < kWarps ? s->items[turn][lane][j] : 0);
  }
  // Over the items i that f takes: of weights, or of ones.
  template <bool kWeights, typename F>
  __device__ __forceinline__ u64 sum_where(const F &f) {
    u64 v[1] = {0};
#pragma unroll
    for (int i = 0; i < kEvery; ++i)
      if (f(i)) v[0] += kWeights ? weight[i] : 1;
    sums<1>(v);
    return v[0];
  }
  // The largest x, of x and any lower bits, for which the sum over the items where f(item) < x is not more than
  // `most`; f takes no item that it is ~0 of.
  template <bool kWeights, typename F>
  __device__ __forceinline__ uint32_t largest(int bits, uint32_t x, u64 most, const F &f) {
    for (int bit = (bits + 1) / 2 * 2 - 2; bit >= 0; bit -= 2) {
      u64 v[3] = {0, 0, 0};
#pragma unroll
      for (int i = 0; i < kEvery; ++i) {
        const uint32_t y = f(i);
        if (y == ~0u) continue;
        const u64 w = kWeights ? weight[i] : 1;
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (y < x + ((uint32_t)(j + 1) << bit)) v[j] += w;
      }
      sums<3>(v);
      x += (uint32_t)((v[0] <= most) + (v[1] <= most) + (v[2] <= most)) << bit;
    }
    return x;
  }
  // The entry at which the sum, in order, reaches `need`; that of all items does.
  template <bool kWeights>
  __device__ u64 reach(u64 need, int id_bits) {
    const auto upper_of = [&](int i) { return (uint32_t)(entry[i] >> 32); };
    uint32_t differ = 0;
#pragma unroll
    for (int i = 0; i < kEvery; ++i)
      if (i * kThreads + (int)threadIdx.x < count) differ |= upper_of(i) ^ s->first;
    differ = __reduce_or_sync(kAll, differ);
    const int lane = threadIdx.x & 31;
    turn ^= 1;
    if (lane == 0) s->items[turn][threadIdx.x >> 5][0] = differ;
    __syncthreads();
    differ = __reduce_or_sync(kAll, lane < kWarps ? (uint32_t)s->items[turn][lane][0] : 0u);
    const int bits = (33 - __clz(differ)) / 2 * 2;
    const uint32_t upper = largest<kWeights>(bits, bits < 32 ? s->first >> bits << bits : 0, need - 1, upper_of);
    const auto equal = [&](int i) { return upper_of(i) == upper; };
    u64 v[2] = {0, 0};  // how many are equal, and what comes before them
#pragma unroll
    for (int i = 0; i < kEvery; ++i) {
      v[0] += equal(i);
      if (upper_of(i) < upper) v[1] += kWeights ? weight[i] : 1;
    }
    sums<2>(v);
    if (v[0] == 1) return (u64)upper << 32 | 0x7FFFFFFFu;
    return (u64)upper << 32 | largest<kWeights>(id_bits, 0, need - 1 - v[1], [&](int i) { return equal(i) ? (uint32_t)entry[i] : ~0u; });
  }
};

// The largest b <= 65535 that at least k of the block's cells reach (0: fewer are that many), of the upper 16
// bits of their keys.
template <int kWarps>
__device__ __forceinline__ uint32_t cell_bound(const uint32_t (&upper)[kEach], int k, Shared *s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t found = 0;
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t mid = found | 1u << bit;
    unsigned mine = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) mine += upper[j] >= mid;
    mine = __reduce_add_sync(kAll, mine);
    if (lane == 0) s->counts[bit & 1][warp] = mine;
    __syncthreads();
    const unsigned all = __reduce_add_sync(kAll, lane < kWarps ? s->counts[bit & 1][lane] : 0u);
    if ((int)all >= k) found = mid;
  }
  return found;
}

// floor(64 t), t below 2^16: the last bits of 2^23 and that.  (A conversion takes four times an addition.)
__device__ __forceinline__ uint32_t step_of(float t) { return __float_as_uint(__fmaf_rd(t, (float)kBinsOfOne, 8388608.0f)) & 0xFFFFu; }

struct Cut {  // tokens are kept from the largest down to this one: key, and id among equal ones
  uint32_t key;
  int id;
  __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= id); }
};

// floor(floor(u 2^31) total / 2^31), total < 2^62.
__device__ __forceinline__ u64 place_of(float u, u64 total) {
  const u64 r = (u64)(u * 2147483648.0f);
  return (total >> 31) * r + (((total & 0x7FFFFFFFull) * r) >> 31);
}

// A row's problem and its steps; every step is called by all threads of the group.
template <typename T, int kThreads>
struct Sampler {
  using R = Row<T>;
  static constexpr int kWarps = kThreads / 32, kShort = 512;
  const SampleArgs &a;
  const R &row;
  Group<kWarps> &g;
  Shared *s;
  u64 *list, *weights, *sums;  // of kList, what is beside it, and the chunks' sums
  float m, c, farthest;
  int index;
  // After find_cut: of what was collected last, the number, where it begins, and the weight and number of all nearer;
  // the chunks' sums are of these.
  int last_count = -1;
  float last_nearest;
  u64 last_above[2];

  __device__ __forceinline__ float t_of(float x) const { return __fmul_rn(__fsub_rn(m, x), c); }
  __device__ __forceinline__ float t_of(u64 entry) const { return t_of(R::value_of(~(uint32_t)(entry >> 32))); }

  __device__ void write(int id, float logprob, int kept) const {
    a.ids[index] = id;
    a.logprob[index] = logprob;
    a.kept[index] = kept;
  }
  // The token at distance t of tokens of `total` together.  The largest one's weight is 2^40, so no part is
  // below 0.
  __device__ void write_token(int id, float t, u64 total, int kept) const {
    write(id, 0.0f - (t * 0.69314718055994531f + log1pf((float)(total - (1ull << 40)) * 0x1p-40f)), kept);
  }

  // The least key with t < bound, of the row's largest or before, sought by a warp's lanes around where it would be without
  // roundings and then between what that leaves; t falls as keys rise.  (Elements are then compared as they are, in bf16
  // by pairs: 608 rows with top_k 1,000 110 -> 97 us, flat rows with top_p 0.95 262 -> 253.)
  __device__ uint32_t first_within(float bound) const {
    uint32_t lo = R::kNothing, hi = R::key(m);  // not so at lo
    const uint32_t near = R::key(m - bound / c) - 16;
    for (bool around = true; hi - lo > 1; around = false) {
      const auto probe = [&](int i) {
        return around ? min(max(near + i, lo), hi) : lo + 1 + (uint32_t)((u64)(hi - lo - 1) * i >> 5);
      };
      const uint32_t yes = __ballot_sync(kAll, t_of(R::value_of(probe(threadIdx.x & 31))) < bound);
      const int first = yes ? __ffs(yes) - 1 : 32;
      const uint32_t above = yes ? probe(first) : hi;
      if (first) lo = probe(first - 1);
      hi = above;
    }
    return hi;
  }

  // Tokens with nearest <= t < beyond into the first block's list; how many there were.  The weights and the number of all
  // tokens with t < near are summed over the group into sum; kChunks: the weights by chunks, too.
  template <bool kSum, bool kChunks>
  __device__ int collect(float nearest, float beyond, float near, u64 (*sum)[2]) {
    const float low = R::value_of(first_within(beyond)), high = nearest > 0.0f ? R::value_of(first_within(nearest) - 1) : m;
    if (threadIdx.x == 0) s->collected = 0;
    g.sync();
    u64 v[2] = {0, 0};
    Weights w;
    for_row(row, g, [&](int chunk, const uint4 (&p)[kEach]) {
      uint32_t found = 0;  // by piece and element
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
#pragma unroll
        for (int e = 0; kSum && e < R::kN; e += 2) {
          const Pair minus = minus_t(R::element(p[j], e), R::element(p[j], e + 1), m, c);
          const float2 t = floats_of(minus);
          w.add(minus, -t.x < near, -t.y < near);
        }
        if (R::value(R::largest(R::none, p[j])) >= low) found |= R::within(p[j], j, low, high);
      }
      if (kSum) {
        const u64 all = w.sum();
        v[0] += all;
        v[1] += w.tokens();
        if (kChunks) put_chunk(chunk, all);
        w = Weights();
      }
      // one addition to the counter for a warp (one for each token took ten times as long as all else)
      if (!__any_sync(kAll, found)) return;
      const int lane = threadIdx.x & 31, mine = __popc(found);
      int before = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(kAll, before, d);
        if (lane >= d) before += y;
      }
      int at = lane == 31 ? atomicAdd(&s->collected, before) : 0;
      at = __shfl_sync(kAll, at, 31) + before - mine;
      for (; found; found &= found - 1, ++at) {
        const int bit = R::place(__ffs(found) - 1), id = row.id(chunk * kChunkPieces + bit / R::kN * 32 + lane) + bit % R::kN;
        if (at < kList) list[at] = (u64)~R::key(row.at(id)) << 32 | (uint32_t)id;
      }
    });
    if (kSum) {
      g.template all<2>(v);
      (*sum)[0] = v[0];
      (*sum)[1] = v[1];
    }
    g.sync();
    int count = s->collected;
    if (g.size > 1) {
      int at[kMaxCluster + 1] = {};
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        int more = 0;
        if (r < g.size) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(more) : "r"(remote(smem_addr(&s->collected), r)) : "memory");
        at[r + 1] = at[r] + more;
      }
      count = at[kMaxCluster];
      if (g.rank == 0 && count <= kList) {
#pragma unroll
        for (int r = 1; r < kMaxCluster; ++r) {
          if ((int)(threadIdx.x >> 5) % kMaxCluster != r || r >= g.size) continue;  // two warps for a block's tokens
          const uint32_t from = remote(smem_addr(list), r);
          for (int i = threadIdx.x / 32 / kMaxCluster * 32 + threadIdx.x % 32; i < at[r + 1] - at[r]; i += kThreads / kMaxCluster) {
            u64 entry;
            asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(entry) : "r"(from + 8u * (uint32_t)i) : "memory");
            list[at[r] + i] = entry;
          }
        }
      }
    }
    __syncthreads();
    if (g.rank == 0 && threadIdx.x == 0 && count > 0 && count <= kList) s->first = (uint32_t)(list[0] >> 32);
    __syncthreads();
    return count;
  }

  __device__ __forceinline__ int id_bits() const { return 32 - __clz(a.vocab); }

  // f of the list's items.
  template <typename F>
  __device__ __forceinline__ void with_items(int count, const F &f) const {
    const auto weight = [&](u64 entry) { return weight_of(t_of(entry)); };
    if (count <= kList / 2) {
      Items<kList / 2 / kThreads, kThreads> items(list, count, s, weight);
      f(items);
    } else {
      Items<kList / kThreads, kThreads> items(list, count, s, weight);
      f(items);
    }
  }

  // draw_from_list for up to kShort tokens, one of a thread's: each against all others, which gives its place and the
  // weight before it, in the order of the tokens and, of those kept, by id.
  __device__ void draw_from_short_list(int count, u64 total) const {
    struct alignas(16) Item {
      u64 entry, weight;
    };
    Item *items = reinterpret_cast<Item *>(weights);
    const int i = threadIdx.x;
    const bool mine = i < count;
    const Item item{mine ? list[i] : ~0ull, mine ? weight_of(t_of(list[i])) : 0};
    if (mine) items[i] = item;
    u64 all[1] = {item.weight};
    sum_in_block(all);
    if (!a.top_k && all[0] < (u64)ceil((double)total * (double)a.top_p)) {
      if (i == 0) {
        s->total = 0;
        s->held = all[0];
      }
      return;
    }
    int place = 0;
    u64 before = 0;
    if (i / 32 * 32 < count)
#pragma unroll 4
      for (int j = 0; j < count; ++j) {
        const Item other = items[j];
        if (other.entry < item.entry) {
          ++place;
          before += other.weight;
        }
      }
    const bool first = mine && (!a.top_k || place < a.top_k);
    u64 v[1] = {first ? item.weight : 0};
    sum_in_block(v);
    if (a.top_k) total = v[0];
    const u64 need = a.top_p < 1.0f ? (u64)ceil((double)total * (double)a.top_p) : 0;
    const bool keep = first && (a.top_p >= 1.0f || before < need) && t_of(item.entry) <= farthest;
    u64 w[2] = {keep ? item.weight : 0, keep};
    sum_in_block(w);
    const u64 at = place_of(a.u[index], w[0]);
    if (keep) items[place] = Item{(uint32_t)item.entry, item.weight};  // all read the old ones before the sums
    __syncthreads();
    if (!keep) return;
    before = 0;
#pragma unroll 4
    for (int j = 0; j < (int)w[1]; ++j)
      if (items[j].entry < (uint32_t)item.entry) before += items[j].weight;
    if (before <= at && at < before + item.weight) {
      write_token((int)(uint32_t)item.entry, t_of(item.entry), w[0], (int)w[1]);
      s->total = 1;
    }
  }
  template <int kM>
  __device__ void sum_in_block(u64 (&v)[kM]) const {
    const int lane = threadIdx.x & 31;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kM; ++j) {
      v[j] = warp_sum(v[j]);
      if (lane == 0) s->items[0][threadIdx.x >> 5][j] = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kM; ++j) v[j] = warp_sum(lane < kWarps ? s->items[0][lane][j] : 0);
  }

  // The first block: cuts the list, which holds all tokens down to some one, and draws from it.  s->total says whether
  // it holds top_p of `total` (0: of its first top_k).
  __device__ void draw_from_list(int count, u64 total) const {
    if (count <= kShort) return draw_from_short_list(count, total);
    with_items(count, [&](auto &items) {
      u64 last = ~0ull;  // of the entries that are kept
      if (a.top_k && a.top_k < count) last = items.template reach<false>((u64)a.top_k, id_bits());
      const auto first = [&](int i) { return items.entry[i] <= last; };
      u64 all = items.template sum_where<true>(first);
      if (a.top_k) total = all;
      const u64 need = a.top_p < 1.0f ? (u64)ceil((double)total * (double)a.top_p) : 0;
      if (need > all) {
        if (threadIdx.x == 0) {
          s->total = 0;
          s->held = all;
        }
        return;
      }
      if (a.top_p < 1.0f) last = min(last, items.template reach<true>(need, id_bits()));
#pragma unroll
      for (int i = 0; i < items.kEvery; ++i)
        if (items.entry[i] > last || !(t_of(items.entry[i]) <= farthest)) items.weight[i] = 0;
      const auto any = [&](int i) { return items.weight[i] != 0; };
      const u64 kept = items.template sum_where<false>(any);
      all = items.template sum_where<true>(any);
      const uint32_t id = items.template largest<true>(id_bits(), 0, place_of(a.u[index], all),
                                                       [&](int i) { return (uint32_t)items.entry[i]; });
      if (threadIdx.x != 0) return;
      write_token((int)id, t_of(row.at((int)id)), all, (int)kept);
      s->total = 1;
    });
  }

  // What the first block put in s->total, in all blocks.
  __device__ __forceinline__ u64 told() {
    g.sync();
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(remote(smem_addr(&s->total), 0)) : "memory");
    g.sync();
    return v;
  }

  // The first block: of the list, the token at which the sum (of weights, or of ones) reaches `need`, into s->total as
  // an entry, all ones where none does; and the sum of all, into s->held.
  template <bool kWeights>
  __device__ void find_in_list(int count, u64 need) const {
    if (count == 0) {
      if (threadIdx.x == 0) {
        s->total = ~0ull;
        s->held = 0;
      }
      return;
    }
    with_items(count, [&](auto &items) {
      const u64 all = items.template sum_where<kWeights>([&](int i) { return i * kThreads + (int)threadIdx.x < count; });
      const u64 entry = all >= need ? items.template reach<kWeights>(need, id_bits()) : ~0ull;
      if (threadIdx.x == 0) {
        s->total = entry;
        s->held = all;
      }
    });
  }

  // The first block: the steps of distance, in s->bins, among whose tokens a sum reaches `need` that is `above` for
  // all tokens nearer than step `from`; and, of ones, the sum before it in s->total.
  template <bool kWeights>
  __device__ void find_steps(const uint32_t *bins, u64 need, int from, u64 above) const {
    constexpr int kOf = (kBins - 1) / kThreads + 1;
    const int first = min(kBins, (int)threadIdx.x * kOf), last = min(kBins, first + kOf);
    const auto mass = [&](int i) { return kWeights ? weight_of((i + 0.5f) / kBinsOfOne) * bins[i] : (u64)bins[i]; };
    u64 mine = 0, all;
    for (int i = first; i < last; ++i) mine += mass(i);
    const u64 begin = block_scan<kWarps>(mine, s, &all);
    u64 before = begin;
    for (int i = first; i < last; ++i) {
      if (i == from) s->total = before;
      before += mass(i);
    }
    if (threadIdx.x == 0) s->bins[0] = s->bins[1] = need > above ? kBins - 1 : 0;
    __syncthreads();
    const u64 sought = s->total + need - above;  // of the sums here, which differ from those that are meant
    __syncthreads();
    before = begin;
    for (int i = first; i < last && (int64_t)sought > 0; ++i) {
      const u64 w = mass(i);
      if (before < sought && sought <= before + w) {
        s->bins[0] = s->bins[1] = i;
        if (!kWeights) s->total = before;
      }
      before += w;
    }
    __syncthreads();
    if (kWeights && threadIdx.x == 0) {  // a step to either side, where the list has room
      const int at = s->bins[0];
      const uint32_t held = bins[at], nearer = at > 0 ? bins[at - 1] : 0, farther = at + 1 < kBins ? bins[at + 1] : 0;
      if (held + nearer + farther <= kList) {
        s->bins[0] = max(at - 1, 0);
        s->bins[1] = min(at + 1, kBins - 1);
      }
    }
    __syncthreads();
  }

  // The cut at the token at which the sum (of weights, or of ones) from the largest down reaches `need`, where the
  // weights, or the tokens at t <= 40, come to that.  Tokens are counted by their distance in steps of 1/64: of
  // ones that gives the step of the cut, and of weights, which differ by 2^(1/64) in a step, one near it from
  // where the sum is known (the first block's `above` for tokens nearer than step `from`).  Its tokens and its
  // neighbours' are collected, and the rest is exact.
  template <bool kWeights>
  __device__ Cut find_cut(u64 need, int from, u64 above) {
    uint32_t *bins = reinterpret_cast<uint32_t *>(weights);
    g.sync();  // the weights were read
    for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
    __syncthreads();
    for_row(row, g, [&](int chunk, const uint4 (&p)[kEach]) {
      for_chunk(row, chunk, p, [&](float x, int) {
        const float t = t_of(x);
        if (t <= kFarthest) atomicAdd(&bins[step_of(t)], 1u);
      });
    });
    g.sync();
    if (g.rank == 0 && g.size > 1) {
      for (int i = threadIdx.x; i < kBins; i += kThreads) {
        uint32_t more[kMaxCluster - 1];
#pragma unroll
        for (int r = 1; r < kMaxCluster; ++r) {
          more[r - 1] = 0;
          if (r < g.size)
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(more[r - 1]) : "r"(remote(smem_addr(bins + i), r)) : "memory");
        }
#pragma unroll
        for (int r = 1; r < kMaxCluster; ++r) bins[i] += more[r - 1];
      }
      __syncthreads();
    }
    for (int turn = 0; turn < 6; ++turn) {
      if (g.rank == 0) find_steps<kWeights>(bins, need, from, above);
      if (!kWeights) above = told();
      else g.sync();
      int bin[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(bin[j]) : "r"(remote(smem_addr(&s->bins[j]), 0)) : "memory");
      const float nearest = (float)bin[0] / kBinsOfOne, beyond = (float)(bin[1] + 1) / kBinsOfOne;
      u64 sum[2] = {0, 0};
      const int count = collect<kWeights, kWeights>(nearest, beyond, nearest, &sum);
      if (kWeights) above = sum[0];
      if (count > kList) break;
      from = bin[0];
      if (kWeights && above >= need) continue;  // the cut is nearer
      if (g.rank == 0) find_in_list<kWeights>(count, need - above);
      const u64 entry = told();
      if (entry != ~0ull) {
        if (kWeights) {
          last_count = count;
          last_nearest = nearest;
          last_above[0] = sum[0];
          last_above[1] = sum[1];
        }
        return Cut{~(uint32_t)(entry >> 32), (int)(uint32_t)entry};
      }
      from = bin[1] + 1;
      if (g.rank == 0) above += s->held;
      g.sync();
    }
    return bracket_cut<kWeights>(need);
  }

  // The same by passes that measure three keys each, however many tokens are equal or nearly so.
  template <bool kWeights>
  __device__ Cut bracket_cut(u64 need) {
    uint32_t lo = R::kNothing + 1, hi = R::key(m) + 1;  // the sum from lo up reaches `need`, from hi up it does not
    u64 above = 0;
    while (hi - lo > 1) {
      uint32_t key[3];
#pragma unroll
      for (int j = 0; j < 3; ++j) key[j] = min(max(hi - (uint32_t)(((u64)(hi - lo) * (j + 1)) >> 2), lo + 1), hi - 1);
      u64 v[3] = {0, 0, 0};
      for_row(row, g, [&](int chunk, const uint4 (&p)[kEach]) {
        for_chunk(row, chunk, p, [&](float x, int) {
          const float t = t_of(x);
          const u64 w = kWeights ? weight_of(t) : t <= kFarthest;
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (R::key(x) >= key[j]) v[j] += w;
        });
      });
      g.template all<3>(v);
      uint32_t new_lo = lo, new_hi = hi;
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        if (v[j] >= need) {
          new_lo = max(new_lo, key[j]);
        } else if (key[j] < new_hi) {
          new_hi = key[j];
          above = v[j];
        }
      }
      lo = new_lo;
      hi = new_hi;
    }
    const u64 w = kWeights ? weight_of(t_of(R::value_of(lo))) : 1;
    id_of_rank(lo, (need - above - 1) / w);
    const u64 entry = told();
    return Cut{~(uint32_t)(entry >> 32), (int)(uint32_t)entry};
  }

  // Sums of chunks into the first block's shared memory.
  __device__ __forceinline__ void put_chunk(int chunk, u64 sum) const {
    sum = warp_sum(sum);
    if ((threadIdx.x & 31) == 0)
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(remote(smem_addr(sums), 0) + 8u * (uint32_t)chunk), "l"(sum) : "memory");
  }
  // The first block: the chunk in which the sum passes `place`, and the sum before it, in s->chunk and s->total.
  __device__ void find_chunk(u64 place) const {
    const int chunks = (row.pieces - 1) / kChunkPieces + 1, per = (chunks - 1) / kThreads + 1;
    const int from = min(chunks, (int)threadIdx.x * per), to = min(chunks, from + per);
    u64 mine = 0, all;
    for (int i = from; i < to; ++i) mine += sums[i];
    if (threadIdx.x == 0) s->chunk = 0;
    u64 before = block_scan<kWarps>(mine, s, &all);
    for (int i = from; i < to; ++i) {
      if (before <= place && place < before + sums[i]) {
        s->chunk = i;
        s->total = before;
      }
      before += sums[i];
    }
    __syncthreads();
  }
  // One warp: the first token of s->chunk at which the sum of f(x, id) passes `place`: then(id, x).
  template <typename F, typename Then>
  __device__ void find_token(u64 place, const F &f, const Then &then) const {
    const int lane = threadIdx.x & 31, first = s->chunk * kChunkPieces + lane;
    uint4 p[kEach];
    u64 before = s->total;
#pragma unroll
    for (int j = 0; j < kEach; ++j) p[j] = row.load(first + j * 32);
#pragma unroll 1
    for (int j = 0; j < kEach; ++j) {
      const uint4 q = j == 0 ? p[0] : j == 1 ? p[1] : j == 2 ? p[2] : p[3];
      u64 mine = 0;
#pragma unroll
      for (int e = 0; e < R::kN; ++e) mine += f(R::element(q, e), row.id(first + j * 32) + e);
      const u64 all = warp_sum(mine);
      if (before <= place && place < before + all) {  // the same in all lanes
        u64 x = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const u64 y = __shfl_up_sync(kAll, x, d);
          if (lane >= d) x += y;
        }
        u64 at = before + x - mine;
        if (at <= place && place < at + mine) {
#pragma unroll
          for (int e = 0; e < R::kN; ++e) {
            const int id = row.id(first + j * 32) + e;
            const u64 w = f(R::element(q, e), id);
            if (at <= place && place < at + w) then(id, R::element(q, e));
            at += w;
          }
        }
        return;
      }
      before += all;
    }
  }

  // The token of this key with so many of lower ids before it, as an entry in the first block's s->total.
  __device__ void id_of_rank(uint32_t key, u64 rank) {
    const auto equal = [&](float x, int) -> u64 { return R::key(x) == key; };
    g.sync();
    for_row(row, g, [&](int chunk, const uint4 (&p)[kEach]) {
      u64 mine = 0;
      for_chunk(row, chunk, p, [&](float x, int id) { mine += equal(x, id); });
      put_chunk(chunk, mine);
    });
    g.sync();
    if (g.rank != 0) return;
    find_chunk(rank);
    u64 entry = 0;
    if (threadIdx.x < 32) {
      bool mine_too = false;
      find_token(rank, equal, [&](int id, float) {
        entry = (u64)~key << 32 | (uint32_t)id;
        mine_too = true;
      });
      __syncwarp();
      if (mine_too) s->total = entry;
    }
    __syncthreads();
  }

  // The weights of a chunk's tokens that keeps(x, t, id) takes.
  template <typename F>
  __device__ __forceinline__ Weights weigh(int chunk, const uint4 (&p)[kEach], const F &keeps) const {
    Weights w;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int id = row.id(chunk * kChunkPieces + j * 32 + (int)(threadIdx.x & 31));
#pragma unroll
      for (int e = 0; e < R::kN; e += 2) {
        const float x = R::element(p[j], e), y = R::element(p[j], e + 1);
        const Pair minus = minus_t(x, y, m, c);
        const float2 t = floats_of(minus);
        w.add(minus, keeps(x, -t.x, id + e), keeps(y, -t.y, id + e + 1));
      }
    }
    return w;
  }

  // draw_from_row after a find_cut that collected the cut's tokens: all nearer ones are kept, and some of these.
  __device__ void draw_from_parts(const Cut &cut) {
    if (g.rank != 0) return;
    u64 v[2] = {0, 0};
    for (int i = threadIdx.x; i < last_count; i += kThreads) {
      const int id = (int)(uint32_t)list[i];
      if (t_of(list[i]) > farthest || !cut.keeps(~(uint32_t)(list[i] >> 32), id)) continue;
      const u64 w = weight_of(t_of(list[i]));
      v[0] += w;
      ++v[1];
      atomicAdd(&sums[(id + row.shift) / R::kN / kChunkPieces], w);
    }
    sum_in_block(v);  // and no sum is added to any more
    const u64 place = place_of(a.u[index], last_above[0] + v[0]);
    draw_at(place, last_above[0] + v[0], (int)(last_above[1] + v[1]),
            [&](float x, float t, int id) { return t <= farthest && cut.keeps(R::key(x), id); });
  }
  // The first block: the token at which the sum, by the chunks' sums and then that of what keeps(x, t, id) takes, passes
  // `place`.
  template <typename F>
  __device__ void draw_at(u64 place, u64 total, int kept, const F &keeps) {
    find_chunk(place);
    if (threadIdx.x < 32)
      find_token(place, [&](float x, int id) { return keeps(x, t_of(x), id) ? weight_of(t_of(x)) : 0; },
                 [&](int id, float x) { write_token(id, t_of(x), total, kept); });
  }

  // Draws from all tokens that the cut and min_p keep.
  template <bool kCut>
  __device__ void draw_from_row(const Cut &cut) {
    const auto keeps = [&](float x, float t, int id) { return t <= farthest && (!kCut || cut.keeps(R::key(x), id)); };
    // Of a chunk whose ids are all up to the cut's, or all past it, tokens above one key are kept.
    const float above = R::value_of(cut.key);
    float from = R::value_of(cut.key - 1);
    if (from == 0.0f) from = R::value_of(cut.key - 2);  // past -0, which is +0
    g.sync();  // the chunks' sums were read
    u64 v[2] = {0, 0};
    for_row(row, g, [&](int chunk, const uint4 (&p)[kEach]) {
      Weights w;
      if constexpr (kCut) {
        const int first = row.id(chunk * kChunkPieces), past = row.id((chunk + 1) * kChunkPieces);
        if (past - 1 <= cut.id || first > cut.id) {
          const float limit = first > cut.id ? above : from;
          w = weigh(chunk, p, [&](float x, float t, int) { return t <= farthest && x > limit; });
        } else {
          w = weigh(chunk, p, keeps);
        }
      } else {
        w = weigh(chunk, p, keeps);
      }
      const u64 sum = w.sum();
      v[0] += sum;
      v[1] += w.tokens();
      put_chunk(chunk, sum);
    });
    g.template all<2>(v);
    g.sync();
    if (g.rank != 0) return;
    draw_at(place_of(a.u[index], v[0]), v[0], (int)v[1], keeps);
  }

  __device__ void run() {
    // the maximum, and those of the cells
    uint32_t cell[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) cell[j] = R::none;
    for_row(row, g, [&](int, const uint4 (&p)[kEach]) {
#pragma unroll
      for (int j = 0; j < kEach; ++j) cell[j] = R::largest(cell[j], p[j]);
    });
    float top = -INFINITY;
    uint32_t upper[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      top = max_nan(top, R::value(cell[j]));
      upper[j] = R::key(R::value(cell[j])) >> (R::kBits - 16);
    }
    u64 v[1] = {isnan(top) ? ~0ull : (u64)R::key(top)};
    g.template all<1, true>(v);
    const float u = a.u[index];
    const bool nothing = v[0] == R::kNothing, wrong = v[0] >= R::kInfinity || !(u >= 0.0f && u < 1.0f);
    if (nothing || wrong) {
      if (g.rank == 0 && threadIdx.x == 0) {
        if (wrong) flag_error(kErrCacheId);
        write(-1, nanf(""), 0);
      }
      return;
    }
    m = R::value_of((uint32_t)v[0]);
    const bool top_k = a.top_k != 0, top_p = a.top_p < 1.0f;
    if (!top_k && !top_p) return draw_from_row<false>(Cut{0, 0});
    // what the cells' bound collects
    const float past = __uint_as_float(__float_as_uint(kFarthest) + 1);
    const int want = top_k ? a.top_k : 128, share = (want - 1) / g.size + 1;
    u64 total = 0, held = 0;  // of the row, and of what was listed, of weights
    int listed = 0;           // the steps of these
    if (share <= kList / 2) {
      u64 least[1] = {0xFFFFull - cell_bound<kWarps>(upper, share, s)};
      g.template all<1, true>(least);
      const uint32_t bound = max((uint32_t)(0xFFFFull - least[0]) << (R::kBits - 16), R::kNothing + 1);
      const float t = t_of(R::value_of(bound));
      const int step = t < kFarthest ? (int)step_of(t) + 1 : kBins;  // whole steps, so that what they hold is known later
      const float beyond = step < kBins ? (float)step / kBinsOfOne : past;
      u64 sum[2] = {0, 0};
      const int count = top_k ? collect<false, false>(0.0f, beyond, 0.0f, nullptr) : collect<true, false>(0.0f, beyond, past, &sum);
      total = sum[0];
      if (count <= kList) {
        if (g.rank == 0) draw_from_list(count, total);
        if (told()) return;
        listed = step;
        if (g.rank == 0) held = s->held;
        g.sync();
      }
    }
    Cut cut{R::kNothing + 1, 0x7FFFFFFF};
    if (top_k) {
      u64 tokens[1] = {0};
      for_row(row, g, [&](int chunk, const uint4 (&p)[kEach]) {
        for_chunk(row, chunk, p, [&](float x, int) { tokens[0] += t_of(x) <= kFarthest; });
      });
      g.template all<1>(tokens);
      if (tokens[0] > (u64)a.top_k) cut = find_cut<false>((u64)a.top_k, 0, 0);
    }
    if (top_p) {
      u64 sum[1] = {total};
      if (top_k) {
        for_row(row, g, [&](int chunk, const uint4 (&p)[kEach]) {
          sum[0] += weigh(chunk, p, [&](float x, float t, int id) { return t <= kFarthest && cut.keeps(R::key(x), id); }).sum();
        });
        g.template all<1>(sum);
      }
      // among the first top_k, whose weight is at least what is needed
      cut = find_cut<true>((u64)ceil((double)sum[0] * (double)a.top_p), listed, held);
    }
    if (top_p && last_count >= 0 && farthest >= last_nearest) draw_from_parts(cut);
    else draw_from_row<true>(cut);
  }
};

constexpr int kSharedBytes = ((int)sizeof(Shared) + 15) / 16 * 16;
template <typename T>
constexpr int smem_of(int vocab) {  // and one chunk more, as a row may begin within a piece
  return kSharedBytes + 8 * (2 * kList + (vocab - 1) / (kChunkPieces * Row<T>::kN) + 2);
}

// kPerSm: blocks that an SM holds, two where rows alone fill the GPU; one has twice the registers.  (All but fp32 with one spill: bf16
// with two 28 bytes of a thread, with one 8 stored and 48 loaded, fp32 with two 8.)
template <typename T, int kThreads, int kPerSm>
__global__ void __launch_bounds__(kThreads, kPerSm) sample_kernel(SampleArgs a, float c, float farthest, int size) {
  extern __shared__ __align__(16) char smem[];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  Shared *s = reinterpret_cast<Shared *>(smem);
  u64 *list = reinterpret_cast<u64 *>(smem + kSharedBytes);
  Group<kThreads / 32> g{size, (int)blockIdx.x % size, 0, s};
  const int index = (int)blockIdx.x / size;
  const Row<T> row(a.logits, a.row, index, a.vocab);
  if (size > 1) g.sync();  // no block writes to one that has not begun
  Sampler<T, kThreads> sampler{a, row, g, s, list, list + kList, list + 2 * kList, 0.0f, c, farthest, index};
  sampler.run();
  if (size > 1) g.sync();  // or to one that has ended
}

template <typename T, int kThreads, int kPerSm>
cudaError_t launch(const SampleArgs &a, int size, cudaStream_t s) {
  constexpr int kMost = smem_of<T>(COPES_MAX_SAMPLE_VOCAB);
  static_assert(kPerSm * (kMost + 1024) <= 228 * 1024, "as many blocks on an SM");
  cudaError_t e = allow_smem((const void *)sample_kernel<T, kThreads, kPerSm>, kMost, kMost);
  if (e != cudaSuccess) return e;
  const float c = a.scale * 1.44269504088896340736f;
  const float farthest = a.min_p > 0.0f ? fminf((float)-log2((double)a.min_p), kFarthest) : kFarthest;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = size;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cfg.stream = s;
  cfg.gridDim = dim3((unsigned)a.n * size);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem_of<T>(a.vocab);
  return cudaLaunchKernelEx(&cfg, sample_kernel<T, kThreads, kPerSm>, a, c, farthest, size);
}

}  // namespace

// Blocks of a row: as many as SMs there are for it.  96 rows of 151,936 in bf16, us with a block on an SM and with two
// blocks of a row, two to an SM, as the kernel was then: uncut 22 and 26, the first 50 17 and 19, top_p of flat rows 98
// and 110.  (1,024 threads on an SM: one row 15.5 instead of 12.7, 96 rows the same.)
template <typename T>
static cudaError_t by_rows(const SampleArgs &a, cudaStream_t s) {
  int size = 1;
  while (size < kMaxCluster && (int64_t)a.n * size * 2 <= 152) size *= 2;
  return a.n <= 152 ? launch<T, 512, 1>(a, size, s) : launch<T, 512, 2>(a, 1, s);
}

cudaError_t launch_sample_tokens(int dtype, const SampleArgs &a, cudaStream_t s) {
  if (a.n == 0) return cudaSuccess;
  g_used = true;
  return dtype == COPES_BF16 ? by_rows<__nv_bfloat16>(a, s) : by_rows<float>(a, s);
}

unsigned read_and_clear_sample_errors() {
  if (!g_used) return 0;
  unsigned v = 0, zero = 0;
  cudaMemcpyFromSymbol(&v, g_sample_error, sizeof(v));
  if (v) cudaMemcpyToSymbol(g_sample_error, &zero, sizeof(zero));
  return v;
}

}  // namespace copes
