// Attention of one new token per sequence over a paged key-value cache.
//
// For a row's query heads h of one key-value head, over its tokens t:
//   s_t = scale q.k_t,  out = sum_t e^(s_t - m) v_t / sum_t e^(s_t - m),  m = max_t s_t.
// Every key and value is read once, for up to 8 or 16 query heads together: 2 flops per value
// and head, 8 flops a byte at 8 heads of bf16.  At the rate of HBM, 6.8 TB/s, that is two thirds of
// the fp32 units' whole rate before a single conversion, and 3% of the tensor cores': the bound is
// HBM, and mma.sync on registers filled from shared memory is enough (tcgen05 takes 64 rows or more
// of one operand; a group of query heads has 1 to 16, and a block of these has no room to wait in).
// Measured: 128 rows of up to 16,384 tokens, 32/8 heads of 128, bf16: 4.24 GB in 605 us, 7.0 TB/s.  Of the
// rate of a copy, 32 rows: bf16 of up to 8,000, 12/4 heads of 192 76%, of 256 86%; fp32 of up to 34,629,
// heads of 80, 94%, of up to 8,000, heads of 192, 75%, of up to 3,000, heads of 256, 51%.
//
// Work.  A row's tokens are cut into tiles; the tiles of all rows and head groups, in one line,
// are shared out evenly among as many blocks as the GPU runs at once, whatever the lengths are.
// The end of a (row, head group) costs about a tile's time and counts as a step of the line, too
// (not where every tile has a block of its own): 32 rows of up to 4,096 tokens took 61 us without
// it, a block with many short rows 67 us where the others took 39.
// A (row, head group) whose tiles lie in several blocks is joined, over the parts in order, by a
// second kernel, whose blocks move in as the first's end (a dependent launch).  (Joined by
// the last of its blocks, counted by an atomic, 60 parts of 16 heads took that block 25 us, and
// few parts 3 us.)
//
// A tile.  Each warp keeps 16 of a tile's tokens to itself, from the copy into shared memory to
// its own running maximum, sum and output, so that the warps need each other only at the end of
// a row.  Where there are rows enough, they do not need each other at all: each warp has a key-value
// head to itself, of as many heads side by side as a block has warps, with tiles of 16 tokens (1,024
// rows of up to 100 tokens: 90 us with the warps on one head, 55 us so; fewer, longer rows would be cut
// into four times the parts).  Keys are the rows of the first product and the query heads its columns,
// S^T[token][head] = K Q^T, and in the second O^T[d][head] = V^T P^T: 8 heads fill a tile of the
// matrix unit, where heads as rows would fill half of 16.  P^T is S^T's registers transposed in
// 8 x 8 blocks (movmatrix).
//
// Precision.  Scores, maxima, sums and outputs are fp32.  bf16: products are exact, and a weight
// p goes into the second product as two bf16 terms (2^-16 of it lost; one term would lose 2^-8
// where the tensor cores have room for both).  The matrix unit cuts its sums where an addition rounds
// them, so a tile's go into a sum of their own, and that by an addition to the row's: continued in the
// matrix unit a row of 131,071 tokens came out 2^-10 of itself too small (the additions cost 6% with heads of
// 192, 4% with 256, 3% with 16 heads on one of the cache's, and nothing else measurable).  fp32: every factor is split into two tf32 terms
// and three of the four products are taken (2^-21 of a product lost at most: that of the small terms,
// 2^-22, and what the splits lose).
#include <math.h>

#include "answer.h"

namespace copes {

__device__ unsigned g_attend_error;
static std::atomic<bool> g_used{false};
__device__ __forceinline__ void flag_error(unsigned bit) { atomicOr(&g_attend_error, bit); }

constexpr int kSMs = 152;
constexpr unsigned kAll = 0xffffffffu;

// What a kernel variant is made of: T of the cache, head_dim padded to DP, NT x 8 query heads, and
// whether the warps of a block have heads side by side or share one.
template <typename T, int DP_, int NT_, bool kBeside>
struct Shape {
  static constexpr bool kFp32 = sizeof(T) == 4;
  static constexpr int DP = DP_, NT = NT_;
  // Warps of a block: what lets the most of them run on an SM.  (fp32 takes twice the room and three
  // times the products.)  Tiles in shared memory: one is worked on while the next is on its way.  With
  // two on their way there is more asked for than HBM can give, and the SMs far from it come to be the
  // last: 128 rows of up to 16,384 tokens took 633 us, 605 so.
  static constexpr int kWarps = !kFp32 ? 4 : DP <= 128 ? 2 : DP <= 192 ? 4 : 3;
  static constexpr int kStages = 2;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kTeam = kBeside ? 1 : kWarps, kSides = kWarps / kTeam;  // warps on a head, heads
  static constexpr int kTile = kTeam * 16;                // tokens
  static constexpr int kChunks = DP * (int)sizeof(T) / 16;  // 16-byte pieces of a token's row
  static constexpr int kPart = 16 * kChunks * 16;         // a warp's keys (or values) of a tile, bytes
  static constexpr int kStage = 2 * kPart * kWarps;
  static constexpr int kHeads = 8 * NT;                   // query heads of a block at a time
  static constexpr int kRow = DP + 4;                     // row of s_o: heads 2j begin 8 banks apart
  static constexpr int kFixed = (kWarps * 8 * kRow + kWarps * 16) * 4;
  static constexpr int kSmem = kStages * kStage + kFixed;
  // blocks of an SM by its 228 KB, 1 KB of them taken for each block, and by its registers
  static constexpr int kFit = 228 * 1024 / (kSmem + 1280);
  // (Three variants spill all the same: fp32 heads of 256 20 bytes of a thread, of 128 with two column
  // tiles 40, of 64 side by side 16.)
  static constexpr int kByRegs = 65536 / (kThreads * (DP > 64 || NT > 1 ? 248 : kFp32 ? 200 : 168));
  static constexpr int kPerSm = kFit < kByRegs ? kFit : kByRegs;
  static_assert(kSmem <= 227 * 1024, "more shared memory than an SM has");
};

// Where a block is in the line of tiles: row by row, key-value head by head, group of query heads
// by group, tile by tile.
struct Cursor {
  int row, tokens, tiles;  // of the row
  int kv, sub, tile;       // kv in kSides; tile >= tiles: a step that stands for the end
};

__device__ __forceinline__ int row_slot(const AttendArgs &a, int row) { return a.slots ? a.slots[row] : row; }

__device__ __forceinline__ int row_tokens(const AttendArgs &a, int slot) {
  return (unsigned)slot < (unsigned)a.c.n_slots ? slot_tokens(a.c, slot) : 0;
}

// The rows after the one that a warp looks tiles up in: their slots and lengths are asked for two and
// one rows before they are used, since a load behind the tiles' copies takes microseconds.
struct RowsAhead {
  int slot, slot1, slot2, length1;  // the row's slot, the next two, the next one's length entry
  __device__ __forceinline__ static int length_of(const AttendArgs &a, int slot) {
    return (unsigned)slot < (unsigned)a.c.n_slots ? a.c.length[slot] : 0;
  }
  __device__ __forceinline__ void begin(const AttendArgs &a, int row) {
    slot = row_slot(a, row);
    slot1 = row + 1 < a.n ? row_slot(a, row + 1) : -1;
    slot2 = row + 2 < a.n ? row_slot(a, row + 2) : -1;
    length1 = length_of(a, slot1);
  }
  __device__ __forceinline__ int next(const AttendArgs &a, int row) {  // moves on to `row`; its tokens
    const int most = a.c.table_width * a.c.page_size, tokens = max(0, min(length1, most));
    slot = slot1;
    slot1 = slot2;
    length1 = length_of(a, slot1);
    slot2 = row + 2 < a.n ? row_slot(a, row + 2) : -1;
    return tokens;
  }
};

// An empty row has one tile, of no tokens, so that somebody writes its output.
template <int kTile>
__device__ __forceinline__ int row_tiles(int tokens) {
  return tokens ? (tokens - 1) / kTile + 1 : 1;
}

// The line shared out: each block has `each` steps, the first `more` of them one more.
struct Shares {
  int each, more;
  __device__ Shares(int total, int blocks) : each(total / blocks), more(total % blocks) {}
  __device__ int begin(int block) const { return block * each + min(block, more); }
  __device__ int owner(int x) const {
    const int longer = more * (each + 1);
    return x < longer ? x / (each + 1) : more + (x - longer) / each;
  }
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Keys and values are read once by a call, and leave L2 first: what else is there stays (parts, tables,
// the program's weights), and of a cache that is read again and again some of its tokens do.  32 rows of up to
// 4,096 tokens, calls on three caches in turn: 42.9 us, 45.6 without; 128 of up to 300 22.6, 24.8.
__device__ __forceinline__ void copy_async(uint32_t to, const void *from, int bytes) {
  uint64_t once;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(once));
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(to), "l"(from), "r"(bytes), "l"(once) : "memory");
}

__device__ __forceinline__ void ldmatrix(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// x in two tf32 terms: hi rounded to nearest, so that x - hi is exact, of either sign and at most 2^-11
// of x's power of two; of it the upper bits (2^-23 of x lost at most, either way).  From 2^128 - 2^116 on
// x would round to infinity, and such values are the caller's not to give: to keep hi finite by
// one more instruction takes 5% longer with heads of 64 to 128 and 16% with 256 (32 rows of up to 3,000: 106 us
// and 123).  The conversion instruction rounds, too, and slowly: 32 fp32 rows of up to 34,629 tokens took
// 329 us with it, 257 so.
__device__ __forceinline__ void split_tf32(uint32_t x, uint32_t &hi, uint32_t &lo) {
  hi = (x + 0x1000u) & 0xFFFFE000u;
  lo = __float_as_uint(__uint_as_float(x) - __uint_as_float(hi)) & 0xFFFFE000u;
}

// c += a b, with both factors in two tf32 terms: the product of the small terms is left out.
__device__ __forceinline__ void mma_split(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  uint32_t ah[4], al[4], bh[2], bl[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) split_tf32(a[i], ah[i], al[i]);
  split_tf32(b0, bh[0], bl[0]);
  split_tf32(b1, bh[1], bl[1]);
  mma_tf32(c, al, bh[0], bh[1]);
  mma_tf32(c, ah, bl[0], bl[1]);
  mma_tf32(c, ah, bh[0], bh[1]);
}

// The same into a sum of its own for each term: three short chains instead of a long one.
__device__ __forceinline__ void mma_split3(float (&c)[3][4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  uint32_t ah[4], al[4], bh[2], bl[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) split_tf32(a[i], ah[i], al[i]);
  split_tf32(b0, bh[0], bl[0]);
  split_tf32(b1, bh[1], bl[1]);
  mma_tf32(c[0], al, bh[0], bh[1]);
  mma_tf32(c[1], ah, bl[0], bl[1]);
  mma_tf32(c[2], ah, bh[0], bh[1]);
}

// A 16-byte piece's place in a row of a tile is its number xor this, so that what one load
// instruction reads lies in different banks.  (Rows of 4 pieces more than a multiple of 8 begin at
// one of two places in the banks, by turns.)
template <typename S>
__device__ __forceinline__ int swizzle(int row) {
  return S::kFp32 ? (row & 6) ^ ((row & 1) << 2) : S::kChunks % 8 ? (row >> 1) & 3 : row & 7;
}

// Factor of a part with maximum m (of log2) in a whole with maximum M.  A part without weight has
// m = -inf and zeros; where its scores are NaN its sums are, and 0 times them still is.
__device__ __forceinline__ float part_weight(float m, float M) { return m == -INFINITY ? 0.0f : exp2_fast(m - M); }

// A warp's state of one (row, head group): heads 8 nt + 2 (lane % 4) + {0, 1}.
template <typename S>
struct Running {
  float m[S::NT][2], l[S::NT][2];     // of log2; l of this lane's tokens alone
  float o[S::DP / 16][S::NT][4];      // O^T: two values of d x two heads each
  __device__ void clear() {
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
      m[j][0] = m[j][1] = -INFINITY;
      l[j][0] = l[j][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < S::DP / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][j][e] = 0.0f;
    }
  }
};

// Query heads as the columns of the first product's second factor.
template <typename S>
struct Queries {
  uint32_t b[S::DP / 16][S::NT][S::kFp32 ? 4 : 2];
};

// `wide`: rows of q are aligned to what a lane loads at a time, 4 bytes of bf16 and 16 of fp32.
template <typename T, typename S>
__device__ __forceinline__ void load_queries(const AttendArgs &a, bool wide, int row, int first_head, int heads,
                                             Queries<S> &q) {
  const int lane = threadIdx.x & 31, D = a.c.head_dim;
#pragma unroll
  for (int j = 0; j < S::NT; ++j) {
    const int h = j * 8 + (lane >> 2);
    const T *from = (const T *)a.q + row * a.q_row + (first_head + h) * a.q_head;
#pragma unroll
    for (int k = 0; k < S::DP / 16; ++k) {
      if constexpr (S::kFp32) {
        // one 16-byte piece of a key's row is the four k of two products: a lane's are d .. d + 3
        const int d = k * 16 + (lane & 3) * 4;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (h < heads && d < D) {
          const uint32_t *u = reinterpret_cast<const uint32_t *>(from + d);
          x = wide ? *reinterpret_cast<const uint4 *>(u) : make_uint4(u[0], u[1], u[2], u[3]);
        }
        q.b[k][j][0] = x.x;
        q.b[k][j][1] = x.y;
        q.b[k][j][2] = x.z;
        q.b[k][j][3] = x.w;
      } else {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int d = k * 16 + (lane & 3) * 2 + e * 8;
          uint32_t x = 0;
          if (h < heads && d < D) {
            const uint16_t *u = reinterpret_cast<const uint16_t *>(from + d);
            x = wide ? *reinterpret_cast<const uint32_t *>(u) : u[0] | (uint32_t)u[1] << 16;
          }
          q.b[k][j][e] = x;
        }
      }
    }
  }
}

// One warp's 16 tokens: scores, the running maximum and sum, and the weighted values.
// `left`: how many of the 16 are tokens.
template <typename S>
__device__ __forceinline__ void warp_tile(uint32_t keys, uint32_t values, int left, float scale, const Queries<S> &q,
                                          Running<S> &r) {
  constexpr int NT = S::NT, KS = S::DP / 16, kPitch = S::kChunks * 16;
  const int lane = threadIdx.x & 31;
  float s[NT][4];
  if constexpr (S::kFp32) {
    constexpr int kSums = NT == 1 ? 2 : 1;  // one for each of the two products of a piece, registers permitting
    float part[NT][kSums][3][4] = {};
    const int row = lane >> 2;
    const uint32_t at = keys + row * kPitch;
    const int x = swizzle<S>(row);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const uint32_t off = (uint32_t)(((k * 4 + (lane & 3)) ^ x) * 16);
      uint32_t u[4], v[4];
      asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "r"(at + off) : "memory");
      asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                   : "r"(at + off + 8 * kPitch) : "memory");
      const uint32_t a0[4] = {u[0], v[0], u[1], v[1]}, a1[4] = {u[2], v[2], u[3], v[3]};
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        mma_split3(part[j][0], a0, q.b[k][j][0], q.b[k][j][1]);
        mma_split3(part[j][kSums - 1], a1, q.b[k][j][2], q.b[k][j][3]);
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float small = part[j][0][0][e] + part[j][0][1][e], large = part[j][0][2][e];
        if constexpr (kSums == 2) {
          small += part[j][1][0][e] + part[j][1][1][e];
          large += part[j][1][2][e];
        }
        s[j][e] = large + small;
      }
  } else {
    float part[NT][2][4] = {};
    const int row = lane & 15, x = swizzle<S>(row);
    const uint32_t at = keys + row * kPitch;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      uint32_t a[4];
      ldmatrix(a, at + (uint32_t)(((k * 2 + (lane >> 4)) ^ x) * 16));
#pragma unroll
      for (int j = 0; j < NT; ++j) mma_bf16(part[j][k & 1], a, q.b[k][j][0], q.b[k][j][1]);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] = part[j][0][e] + part[j][1][e];
  }

  // tokens lane / 4 (s[.][0], s[.][1]) and lane / 4 + 8
  const bool here[2] = {(lane >> 2) < left, (lane >> 2) + 8 < left};
  bool grown = false;
  float keep[NT][2];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      s[j][e] = here[0] ? s[j][e] * scale : -INFINITY;
      s[j][2 + e] = here[1] ? s[j][2 + e] * scale : -INFINITY;
      float top = fmaxf(s[j][e], s[j][2 + e]);
      top = fmaxf(top, __shfl_xor_sync(kAll, top, 4));
      top = fmaxf(top, __shfl_xor_sync(kAll, top, 8));
      top = fmaxf(top, __shfl_xor_sync(kAll, top, 16));
      const float m = fmaxf(r.m[j][e], top);
      keep[j][e] = m == r.m[j][e] ? 1.0f : exp2_fast(r.m[j][e] - m);
      grown |= m != r.m[j][e];
      r.m[j][e] = m;
      const float base = m == -INFINITY ? 0.0f : m;
      s[j][e] = exp2_fast(s[j][e] - base);
      s[j][2 + e] = exp2_fast(s[j][2 + e] - base);
      r.l[j][e] = r.l[j][e] * keep[j][e] + (s[j][e] + s[j][2 + e]);
    }
  if (__any_sync(kAll, grown)) {
#pragma unroll
    for (int i = 0; i < KS; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) r.o[i][j][e] *= keep[j][e & 1];
  }

  if constexpr (S::kFp32) {
    // P^T: 8 tokens x 8 heads at a time, in 16-bit halves.  A lane then has tokens 2j and 2j + 1
    // (j = lane % 4) as the k of one product: its values are read from those rows.
    uint32_t p[NT][2][2];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t u = __float_as_uint(s[j][2 * e]), v = __float_as_uint(s[j][2 * e + 1]);
        const uint32_t lo = transpose8(__byte_perm(u, v, 0x5410)), hi = transpose8(__byte_perm(u, v, 0x7632));
        p[j][e][0] = __byte_perm(lo, hi, 0x5410);
        p[j][e][1] = __byte_perm(lo, hi, 0x7632);
      }
#pragma unroll
    for (int g = 0; g < S::DP / 32; ++g) {
      float sum[2][NT][4] = {};  // of the tile
      const int piece = g * 8 + (lane >> 2);  // d = 32 g + 4 (lane / 4) + 0 .. 3
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = e * 8 + (lane & 3) * 2;
        const uint32_t at = values + row * kPitch;
        uint32_t u[4], v[4];
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                     : "r"(at + (uint32_t)((piece ^ swizzle<S>(row)) * 16)) : "memory");
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                     : "r"(at + kPitch + (uint32_t)((piece ^ swizzle<S>(row + 1)) * 16)) : "memory");
        const uint32_t a0[4] = {u[0], u[1], v[0], v[1]}, a1[4] = {u[2], u[3], v[2], v[3]};
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          mma_split(sum[0][j], a0, p[j][e][0], p[j][e][1]);
          mma_split(sum[1][j], a1, p[j][e][0], p[j][e][1]);
        }
      }
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          r.o[2 * g][j][e] += sum[0][j][e];
          r.o[2 * g + 1][j][e] += sum[1][j][e];
        }
    }
  } else {
    uint32_t p[NT][2], rest[NT][2];  // tokens 0 .. 7 and 8 .. 15, in two bf16 terms
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float u = s[j][2 * e], v = s[j][2 * e + 1];
        const uint32_t hi = pack_bf16(u, v);
        p[j][e] = transpose8(hi);
        rest[j][e] = transpose8(pack_bf16(u - __uint_as_float(hi << 16), v - __uint_as_float(hi & 0xFFFF0000u)));
      }
    const int row = (lane & 7) + (lane >> 4) * 8, x = swizzle<S>(row);
    const uint32_t at = values + row * kPitch;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      uint32_t a[4];
      ldmatrix_trans(a, at + (uint32_t)(((i * 2 + ((lane >> 3) & 1)) ^ x) * 16));
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float sum[4] = {};  // of the tile
        mma_bf16(sum, a, rest[j][0], rest[j][1]);
        mma_bf16(sum, a, p[j][0], p[j][1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) r.o[i][j][e] += sum[e];
      }
    }
  }
}

// The d of r.o[i][.][2 half + .].
template <typename S>
__device__ __forceinline__ int output_d(int i, int half) {
  const int lane = threadIdx.x & 31;
  return S::kFp32 ? (i >> 1) * 32 + (lane >> 2) * 4 + (i & 1) * 2 + half : i * 16 + (lane >> 2) + half * 8;
}

__device__ __forceinline__ void store(float4 x, float *to) { *reinterpret_cast<float4 *>(to) = x; }
__device__ __forceinline__ void store(float4 x, __nv_bfloat16 *to) {
  *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
}
__device__ __forceinline__ void fma4(float4 &o, float f, const float4 &x) {
  o.x = fmaf(f, x.x, o.x);
  o.y = fmaf(f, x.y, o.y);
  o.z = fmaf(f, x.z, o.z);
  o.w = fmaf(f, x.w, o.w);
}
// o / L, 0 of an empty row.
__device__ __forceinline__ float4 normalised(const float4 &o, float L) {
  const float f = L == 0.0f ? 0.0f : 1.0f / L;
  return make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
}
__device__ __forceinline__ float log_sum(float M, float L) {
  return L == 0.0f ? -INFINITY : fmaf(0.6931471805599453094f, M, logf(L));
}

// t / d by a product: t < 2^31, m = ceil(2^(31 + s) / d) with 2^s >= d, so m d = 2^(31 + s) + e with
// e < 2^s, and t e < 2^(31 + s) adds nothing to the quotient.
struct Divisor {
  uint32_t m;
  int s;
  __host__ explicit Divisor(uint32_t d) : s(0) {
    while ((1ull << s) < d) ++s;
    m = (uint32_t)(((1ull << (31 + s)) + d - 1) / d);
  }
  __device__ __forceinline__ int quotient(int t) const { return (int)(((uint64_t)(uint32_t)t * m) >> (31 + s)); }
};

// The workspace: a Split for every block, then the parts: block w's at 2 w (of a row that begins
// before the block's share) and 2 w + 1 (of one that ends after it), each for kSides heads kHeads
// maxima, kHeads sums and kHeads x head_dim values.
struct alignas(16) Split {  // what begins in block w's share and goes on to that of block `last`; row -1: nothing
  int row, kv, sub, last;
};

template <typename T, typename S>
__global__ void __launch_bounds__(S::kThreads, S::kPerSm) attend_kernel(AttendArgs a, Split *split, float *part,
                                                                        int groups, Divisor by_page) {
  extern __shared__ __align__(128) char smem[];
  __shared__ Cursor s_at;
  __shared__ int s_sum[S::kWarps];
  constexpr int TILE = S::kTile, kTeamThreads = S::kTeam * 32;
  const Cache &c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, D = c.head_dim;
  // this warp's head beside the others', its place among the warps on that head, and this thread's
  const int side = warp / S::kTeam, member = warp % S::kTeam, rank = tid % kTeamThreads;
  const int group = a.q_heads / c.n_kv_heads, beside = c.n_kv_heads / S::kSides, units = beside * groups;
  const auto team_sync = [] {
    if constexpr (S::kTeam == 1) __syncwarp();
    else __syncthreads();
  };

  // Launched while the kernel before it on the stream ends, whose results are waited for here (32 rows of
  // up to 4,096 tokens, call after call: 47.0 us, and 49.6 where each launch waits for the last one's end).
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // The line's length and this block's share [lo, hi) of it: a thread adds up a few rows in order.
  // Their tiles wait where the keys and values will be, if there is room, or are counted twice.
  int *s_tiles = reinterpret_cast<int *>(smem);
  const bool kept = a.n <= S::kStages * S::kStage / 4;
  const auto tiles_of = [&](int i) { return kept ? s_tiles[i] : row_tiles<TILE>(row_tokens(a, row_slot(a, i))); };
  if (kept) {
    for (int i = tid; i < a.n; i += S::kThreads) s_tiles[i] = row_tiles<TILE>(row_tokens(a, row_slot(a, i)));
    __syncthreads();
  }
  const int rows = (a.n + S::kThreads - 1) / S::kThreads, r0 = min(a.n, tid * rows), r1 = min(a.n, r0 + rows);
  int mine = 0;
  for (int i = r0; i < r1; ++i) mine += tiles_of(i);
  int before = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(kAll, before, d);
    if (lane >= d) before += y;
  }
  if (lane == 31) s_sum[warp] = before;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < S::kWarps; ++w) {
    if (w < warp) before += s_sum[w];
    total += s_sum[w];
  }
  const int ends = total * units > (int)gridDim.x ? S::NT : 0;  // steps that an end counts for
  before += r0 * ends - mine;
  mine += (r1 - r0) * ends;
  total = (total + a.n * ends) * units;
  const int blocks = min((int)gridDim.x, total);  // each has a step at least
  if (blockIdx.x >= blocks) {
    if (tid == 0) split[blockIdx.x] = Split{-1, 0, 0, 0};
    return;
  }
  const Shares shares(total, blocks);
  const int lo = shares.begin(blockIdx.x), count = shares.begin(blockIdx.x + 1) - lo;
  if (before * units <= lo && lo < (before + mine) * units) {
    Cursor at;
    at.row = r0;
    for (;; ++at.row) {
      at.tiles = tiles_of(at.row);
      if (at.row + 1 >= r1 || lo < (before + at.tiles + ends) * units) break;
      before += at.tiles + ends;
    }
    at.tokens = row_tokens(a, row_slot(a, at.row));
    const int unit = (lo - before * units) / (at.tiles + ends);
    at.tile = (lo - before * units) % (at.tiles + ends);
    at.kv = unit / groups;
    at.sub = unit % groups;
    s_at = at;
  }
  __syncthreads();
  Cursor at = s_at, ahead = at;
  RowsAhead rows_ahead;
  rows_ahead.begin(a, at.row);
  if (tid == 0 && (unsigned)rows_ahead.slot >= (unsigned)c.n_slots) flag_error(kErrCacheId);
  // The tokens of the rows between `at` and `ahead`, by row % 8: the cursors are at most kStages + 2
  // steps, and so rows, apart (two look-ups before the first tile is asked for, one with each).
  static_assert(S::kStages + 2 < 8, "a lane for each row between the cursors");
  int tokens_of_row = 0;
  // the next (row, head group); true where that is another row
  const auto next_unit = [&](Cursor &x) {
    x.tile = 0;
    if (++x.sub < groups) return false;
    x.sub = 0;
    if (++x.kv < beside) return false;
    x.kv = 0;
    ++x.row;
    return true;
  };
  const auto advance_ahead = [&]() {
    if (++ahead.tile < ahead.tiles + ends || !next_unit(ahead) || ahead.row >= a.n) return;
    ahead.tokens = rows_ahead.next(a, ahead.row);
    ahead.tiles = row_tiles<TILE>(ahead.tokens);
    if (tid == 0 && (unsigned)rows_ahead.slot >= (unsigned)c.n_slots) flag_error(kErrCacheId);
    if (lane == (ahead.row & 7)) tokens_of_row = ahead.tokens;
  };
  const auto advance_at = [&]() {
    if (++at.tile < at.tiles + ends || !next_unit(at) || at.row >= a.n) return;
    at.tokens = __shfl_sync(kAll, tokens_of_row, at.row & 7);
    at.tiles = row_tiles<TILE>(at.tokens);
  };

  float *s_o = reinterpret_cast<float *>(smem + S::kStages * S::kStage);  // [warp][8][kRow]
  float *s_m = s_o + S::kWarps * 8 * S::kRow + side * S::kTeam * 8, *s_l = s_m + S::kWarps * 8;
  s_o += side * S::kTeam * 8 * S::kRow;  // of the warps on this head, like s_m and s_l
  const uint32_t stages = smem_addr(smem) + warp * 2 * S::kPart;
  const uint64_t head_bytes = (uint64_t)c.head_elems * sizeof(T), to_values = c.n_kv_heads * head_bytes;
  const char *pool = c.pool + (uint64_t)a.layer * c.layer_elems * sizeof(T) + side * head_bytes;

  // Where token (16 member + lane % 16) of a tile is: its page (-1 for none, -2 for one outside the
  // pool), its place there and the tile's key-value head.  Tables are read two tiles ahead of the
  // tile that is asked for, so that nothing waits for them.
  struct Place {
    int page, place, kv;
  };
  int looked = 0;
  const auto look_up = [&]() {
    Place p{-1, 0, ahead.kv};
    if (looked == count) return p;
    const int t = ahead.tile * TILE + member * 16 + (lane & 15);
    if (ahead.tile < ahead.tiles && t < ahead.tokens) {
      const int at_page = by_page.quotient(t);
      p.place = t - at_page * c.page_size;
      p.page = c.table[(int64_t)rows_ahead.slot * c.table_width + at_page];
      if ((unsigned)p.page >= (unsigned)c.n_pages) p.page = -2;
    }
    if (++looked < count) advance_ahead();
    return p;
  };
  const auto ask = [&](int stage, const Place &p) {
    if (!__any_sync(kAll, p.page != -1)) return;  // nothing of this warp's is read
    const char *from = nullptr;
    if (p.page >= 0) from = pool + (uint64_t)p.page * c.page_bytes + p.kv * S::kSides * head_bytes + (uint64_t)p.place * D * sizeof(T);
    else if (p.page == -2) flag_error(kErrCacheId);
    const uint32_t to = stages + stage * S::kStage;
#pragma unroll
    for (int i = 0; i < S::kChunks / 2; ++i) {
      const int row = (i * 32 + lane) / S::kChunks, piece = (i * 32 + lane) % S::kChunks;
      const char *src = reinterpret_cast<const char *>(__shfl_sync(kAll, (unsigned long long)from, row));
      const int bytes = src && piece * 16 < D * (int)sizeof(T) ? 16 : 0;  // 0: zeros
      src = bytes ? src + piece * 16 : c.pool;
      const uint32_t dst = to + (row * S::kChunks + (piece ^ swizzle<S>(row))) * 16;
      copy_async(dst, src, bytes);
      copy_async(dst + S::kPart, bytes ? src + to_values : src, bytes);
    }
  };
  Place next = look_up();
  // The queries of a (row, head group), and, registers permitting, of the next one, asked for a
  // (row, head group) before they are used.
  constexpr bool kNextToo = S::NT == 1 && (S::kFp32 ? S::DP <= 64 : S::DP <= 128);
  const int64_t q_bytes = sizeof(T), q_wide = S::kFp32 ? 16 : 4;
  const bool wide = (uintptr_t)a.q % q_wide == 0 && a.q_row * q_bytes % q_wide == 0 && a.q_head * q_bytes % q_wide == 0;
  Queries<S> q, q_next;
  const auto queries_of = [&](const Cursor &x, Queries<S> &to) {
    if (x.row < a.n)
      load_queries<T, S>(a, wide, x.row, (x.kv * S::kSides + side) * group + x.sub * S::kHeads,
                         min(S::kHeads, group - x.sub * S::kHeads), to);
  };
  Cursor asking = at;  // whose queries were asked for last
  if (at.tile >= at.tiles) next_unit(asking);
  queries_of(asking, q);
  if constexpr (kNextToo) {
    next_unit(asking);
    if (count > at.tiles - at.tile) queries_of(asking, q_next);
  }
  Place after = look_up();

  int asked = 0;
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s) {
    if (asked < count) {
      ask(s, next);
      ++asked;
      next = after;
      after = look_up();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }

  Running<S> r;
  r.clear();
  const float scale = a.scale * 1.44269504088896340736f;  // of log2
  constexpr int kD4 = S::DP / 4;
  const int slot_floats = S::kHeads * (D + 2);
  Split begun{-1, 0, 0, 0};
  for (int j = 0; j < count; ++j) {
    if (asked < count) {
      ask(asked % S::kStages, next);
      ++asked;
      next = after;
      after = look_up();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 1) : "memory");
    __syncwarp();
    const int left = at.tile < at.tiles ? at.tokens - at.tile * TILE - member * 16 : 0;
    const uint32_t tile = stages + j % S::kStages * S::kStage;
    if (left > 0) warp_tile<S>(tile, tile + S::kPart, left, scale, q, r);
    __syncwarp();

    const Cursor was = at;
    if (j + 1 < count) advance_at();
    if (was.tile >= was.tiles || (was.tile + 1 < was.tiles && j + 1 < count)) continue;
    if (j + 1 + ends < count) {
      if constexpr (kNextToo) q = q_next;
      next_unit(asking);
      queries_of(asking, kNextToo ? q_next : q);
    }

    // the warps' states together
    const int x0 = lo + j - was.tile, x1 = x0 + was.tiles - 1;
    const bool whole = lo <= x0 && x1 < lo + count;
    const int first_head = (was.kv * S::kSides + side) * group + was.sub * S::kHeads;
    const int heads = min(S::kHeads, group - was.sub * S::kHeads);
    float *mine_part = part + ((int64_t)(2 * (int)blockIdx.x + (lo > x0 ? 0 : 1)) * S::kSides + side) * slot_floats;
    const int64_t first = (int64_t)was.row * a.q_heads + first_head;
#pragma unroll
    for (int nt = 0; nt < S::NT; ++nt) {
      team_sync();  // s_o may still be read
      float factor[2] = {1.0f, 1.0f};  // a warp alone normalises its values on their way to s_o
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float l = r.l[nt][e];
        l += __shfl_xor_sync(kAll, l, 4);
        l += __shfl_xor_sync(kAll, l, 8);
        l += __shfl_xor_sync(kAll, l, 16);
        const int h = lane * 2 + e;
        if constexpr (S::kTeam > 1) {
          if (lane < 4) {
            s_m[member * 8 + h] = r.m[nt][e];
            s_l[member * 8 + h] = l;
          }
        } else {
          if (whole) factor[e] = l == 0.0f ? 0.0f : 1.0f / l;
          if (lane < 4 && nt * 8 + h < heads) {
            if (!whole) {
              mine_part[nt * 8 + h] = r.m[nt][e];
              mine_part[S::kHeads + nt * 8 + h] = l;
            } else if (a.lse) {
              a.lse[first + nt * 8 + h] = log_sum(r.m[nt][e], l);
            }
          }
        }
      }
#pragma unroll
      for (int i = 0; i < S::DP / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s_o[(member * 8 + (lane & 3) * 2 + (e & 1)) * S::kRow + output_d<S>(i, e >> 1)] = r.o[i][nt][e] * factor[e & 1];
      team_sync();
      for (int v = rank; v < 8 * kD4; v += kTeamThreads) {
        const int h = v / kD4, d = v % kD4 * 4;
        if (nt * 8 + h >= heads || d >= D) continue;
        float4 o;
        if constexpr (S::kTeam > 1) {
          float M = -INFINITY, L = 0.0f;
#pragma unroll
          for (int w = 0; w < S::kTeam; ++w) M = fmaxf(M, s_m[w * 8 + h]);
          o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int w = 0; w < S::kTeam; ++w) {
            const float weight = part_weight(s_m[w * 8 + h], M);
            L = fmaf(weight, s_l[w * 8 + h], L);
            fma4(o, weight, *reinterpret_cast<const float4 *>(s_o + (w * 8 + h) * S::kRow + d));
          }
          if (whole) o = normalised(o, L);
          if (d == 0 && !whole) {
            mine_part[nt * 8 + h] = M;
            mine_part[S::kHeads + nt * 8 + h] = L;
          } else if (d == 0 && a.lse) {
            a.lse[first + nt * 8 + h] = log_sum(M, L);
          }
        } else {
          o = *reinterpret_cast<const float4 *>(s_o + h * S::kRow + d);
        }
        if (whole) store(o, (T *)a.out + (first + nt * 8 + h) * D + d);
        else *reinterpret_cast<float4 *>(mine_part + 2 * S::kHeads + (nt * 8 + h) * D + d) = o;
      }
    }
    if (!whole && lo <= x0) begun = Split{was.row, was.kv, was.sub, shares.owner(x1)};
    r.clear();
  }

  if (tid == 0) split[blockIdx.x] = begun;
}

// Joins the parts of what begins in one block's share and goes on in others: `per` blocks for each
// block of attend_kernel, one for a query head (of the kheads that a part has room for) of all `sides`
// heads beside one another.  Warps (pairs of them for more than 128 components) take the sides and
// the parts by turns, kBatch of them on their way at once.
// Most blocks find nothing to join, and all that the SMs hold wait there for attend_kernel's end, so
// there are to be many of them on an SM: 1,216 blocks took 9 us with the 80 registers of a batch of
// 8, which only few rows in many parts want.  (In the 40 of a batch of 4 28 bytes are spilled.)
constexpr int kJoinThreads = 256;
template <typename T, int kBatch>
__global__ void __launch_bounds__(kJoinThreads, kBatch > 4 ? 3 : 6) join_kernel(AttendArgs a, const Split *split,
                                                                              const float *part, int kheads, int per,
                                                                              int sides) {
  __shared__ float4 s_o[kJoinThreads];
  __shared__ float s_m[kJoinThreads / 32], s_l[kJoinThreads / 32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int w0 = blockIdx.x / per, h = blockIdx.x % per, D = a.c.head_dim;
  const Split x = split[w0];
  const int group = a.q_heads / a.c.n_kv_heads;
  if (x.row < 0 || h >= min(kheads, group - x.sub * kheads)) return;
  const int wide = D > 128 ? 64 : 32, mine = threadIdx.x / wide, turns = kJoinThreads / wide / sides;
  const int d = threadIdx.x % wide * 4, slot_floats = kheads * (D + 2);
  float M = -INFINITY, L = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int w = w0 + mine / sides; w <= x.last; w += turns * kBatch) {
    float m[kBatch], l[kBatch];
    float4 y[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int from = w + u * turns;
      m[u] = -INFINITY;
      l[u] = 0.0f;
      y[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (from <= x.last) {
        const float *p = part + ((int64_t)(2 * from + (from == w0 ? 1 : 0)) * sides + mine % sides) * slot_floats;
        m[u] = p[h];
        l[u] = p[kheads + h];
        if (d < D) y[u] = *reinterpret_cast<const float4 *>(p + 2 * kheads + h * D + d);
      }
    }
    float N = M;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) N = fmaxf(N, m[u]);
    const float keep = part_weight(M, N);
    L *= keep;
    o = make_float4(o.x * keep, o.y * keep, o.z * keep, o.w * keep);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float weight = part_weight(m[u], N);
      L = fmaf(weight, l[u], L);
      fma4(o, weight, y[u]);
    }
    M = N;
  }
  s_o[threadIdx.x] = o;
  if (threadIdx.x % wide == 0) {
    s_m[mine] = M;
    s_l[mine] = L;
  }
  __syncthreads();
  if (mine >= sides || d >= D) return;  // the first turns of the sides go on
  M = -INFINITY;
  L = 0.0f;
  o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int t = 0; t < turns; ++t) M = fmaxf(M, s_m[t * sides + mine]);
  for (int t = 0; t < turns; ++t) {
    const float weight = part_weight(s_m[t * sides + mine], M);
    L = fmaf(weight, s_l[t * sides + mine], L);
    fma4(o, weight, s_o[t * sides * wide + threadIdx.x]);
  }
  const int64_t head = (int64_t)x.row * a.q_heads + (x.kv * sides + mine) * group + x.sub * kheads + h;
  store(normalised(o, L), (T *)a.out + head * D + d);
  if (d == 0 && a.lse) a.lse[head] = log_sum(M, L);
}

namespace {

template <typename T, int DP, int NT, bool kBeside>
cudaError_t launch(const AttendArgs &a, void *ws, cudaStream_t s, size_t *bytes) {
  using S = Shape<T, DP, NT, kBeside>;
  const int group = a.q_heads / a.c.n_kv_heads, groups = (group + S::kHeads - 1) / S::kHeads;
  // blocks that the GPU runs at once, or fewer where the tables have no room for so many tiles
  const int64_t room = (int64_t)a.c.table_width * a.c.page_size, tiles = (room + S::kTile - 1) / S::kTile;
  const int64_t most = (int64_t)a.n * (a.c.n_kv_heads / S::kSides) * groups * tiles;
  const unsigned blocks = (unsigned)(most < kSMs * S::kPerSm ? most : kSMs * S::kPerSm);
  if (bytes) {
    *bytes = blocks * sizeof(Split) + (size_t)2 * blocks * S::kSides * S::kHeads * (a.c.head_dim + 2) * 4;
    return cudaSuccess;
  }
  cudaError_t e = allow_smem((const void *)attend_kernel<T, S>, S::kSmem, S::kSmem);
  if (e != cudaSuccess) return e;
  Split *split = (Split *)ws;
  float *part = (float *)(split + blocks);
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cfg.stream = s;
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(S::kThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  e = cudaLaunchKernelEx(&cfg, attend_kernel<T, S>, a, split, part, groups, Divisor(a.c.page_size));
  if (e != cudaSuccess || tiles <= 1) return e;  // of one tile nothing is split
  const int per = S::kHeads < group ? S::kHeads : group;
  cfg.gridDim = dim3(blocks * per);
  cfg.blockDim = dim3(kJoinThreads);
  cfg.dynamicSmemBytes = 0;
  // Batches of 8 parts where a row has many (us with 8 and with 4; 16/1 heads of 128, bf16: 1 row of 20,000 tokens 20.9,
  // 37.3, 32 of up to 4,000 19.9, 17.7; 14/2 heads of 64: 1 row of 20,000 15.3, 19.0, 16 of up to 8,000 15.5, 14.2).  Near the
  // bound it takes 8 where 4 suits better: 8 rows of up to 4,000 of the former 14.4, 13.1, of up to 8,000 of the latter 13.1, 12.4.
  const auto join = blocks >= 16 * (int64_t)a.n * a.c.n_kv_heads * groups ? join_kernel<T, 8> : join_kernel<T, 4>;
  return cudaLaunchKernelEx(&cfg, join, a, (const Split *)split, (const float *)part, S::kHeads, per, S::kSides);
}

// Heads side by side where there are three rows' for four of the blocks that run at once.  32/8 heads, us
// on one head and side by side (* what the rule takes), rows of up to 300 tokens, and of up to 3,000:
//                40 rows       120           160           480           960             120 (3,000)
//   bf16  64     10.8* 11.8    16.7* 16.5    20.6* 19.9    42.3 37.2*    74.8 59.0*      65.0* 62.1
//         96     12.0* 13.2    21.4 22.0*    27.0 25.8*    61.2 50.6*    113.7 83.1*     93.4 88.5*
//         128    12.7* 14.1    23.1 22.9*    29.2 27.1*    67.3 56.6*    126.3 97.6*     114.4 114.3*
//   fp32  64     14.7* 15.0    25.9* 26.0    31.8 31.2*    70.7 67.1*    130.1 120.0*    130.0* 126.7
//         96     16.8* 16.2    29.8 28.9*    36.2 35.0*    83.1 78.2*    155.1 142.7*    166.7 171.1*
//         128    19.8* 18.5    38.3 36.0*    47.6 44.6*    119.0 107.3*   225.3 203.1*   231.8 228.0*
// and 1,024 rows of up to 100 (bf16, 128) 90, 52.
template <typename T, int DP>
cudaError_t one_group(const AttendArgs &a, void *ws, cudaStream_t s, size_t *bytes) {
  using S = Shape<T, DP, 1, true>;
  if (a.c.n_kv_heads % S::kSides == 0 && (int64_t)a.n * (a.c.n_kv_heads / S::kSides) * 4 >= 3 * kSMs * S::kPerSm)
    return launch<T, DP, 1, true>(a, ws, s, bytes);
  return launch<T, DP, 1, false>(a, ws, s, bytes);
}

// Up to 8 query heads of a key-value head at a time, or 16 where it has more (each further group
// reads the keys and values again); 8 for head_dim past 128, whose state would not fit in
// registers twice.
template <typename T>
cudaError_t by_shape(const AttendArgs &a, void *ws, cudaStream_t s, size_t *bytes) {
  const bool many = a.q_heads / a.c.n_kv_heads > 8;
  if (a.c.head_dim <= 64) return many ? launch<T, 64, 2, false>(a, ws, s, bytes) : one_group<T, 64>(a, ws, s, bytes);
  if (a.c.head_dim <= 96) return many ? launch<T, 96, 2, false>(a, ws, s, bytes) : one_group<T, 96>(a, ws, s, bytes);
  if (a.c.head_dim <= 128) return many ? launch<T, 128, 2, false>(a, ws, s, bytes) : one_group<T, 128>(a, ws, s, bytes);
  if (a.c.head_dim <= 192) return launch<T, 192, 1, false>(a, ws, s, bytes);
  return launch<T, 256, 1, false>(a, ws, s, bytes);
}

cudaError_t dispatch(int dtype, const AttendArgs &a, void *ws, cudaStream_t s, size_t *bytes) {
  return dtype == COPES_BF16 ? by_shape<__nv_bfloat16>(a, ws, s, bytes) : by_shape<float>(a, ws, s, bytes);
}

}  // namespace

size_t attend_workspace_bytes(const Cache &c, int n, int q_heads) {
  AttendArgs a{};
  a.c = c;
  a.n = n;
  a.q_heads = q_heads;
  size_t bytes = 0;
  dispatch(c.elem == 2 ? COPES_BF16 : COPES_FP32, a, nullptr, 0, &bytes);
  return bytes ? bytes : 16;
}

cudaError_t launch_paged_attention(int dtype, const AttendArgs &a, void *ws, cudaStream_t s) {
  if (a.n == 0) return cudaSuccess;
  g_used = true;
  return dispatch(dtype, a, ws, s, nullptr);
}

unsigned read_and_clear_attend_errors() {
  if (!g_used) return 0;
  unsigned v = 0, zero = 0;
  cudaMemcpyFromSymbol(&v, g_attend_error, sizeof(v));
  if (v) cudaMemcpyToSymbol(g_attend_error, &zero, sizeof(zero));
  return v;
}

}  // namespace copes
