// The residual sum of a block with the norms before and after it, a row at a time.
//
// With rms(a) = sqrt(mean a^2 + eps), g a gate and c the residual scale:
//   z = y / rms(y) out_weight (or y),   s = x + (c g) z,   normed = s / rms(s) weight.
// A row's values stay in the registers of its threads from the one read to the one write, so each
// array passes HBM once, and HBM bounds it where there are many rows: 16,384 of 4,096 in bf16, with a norm after the
// block and a gate for every channel, 537 MB in 99 us, 5.4 TB/s, four fifths of a copy's rate (of the issue slots,
// two thirds: a value's way from bf16 and back takes as many operations as the sums).  A few rows are a chain of a load, two
// sums over the row's threads and a store: one row of 896 2.2 us, 22,400 rows of 128 (the norm alone) 4.2, 301 rows of 2,561
// in fp32 that begin anywhere 8.6.
#include <float.h>
#include <math.h>

#include "answer.h"
#include "copes_device.cuh"

namespace copes {

constexpr unsigned kAll = 0xffffffffu;

// kBytes of T: a piece of a row, as it is in memory.
template <typename T, int kBytes>
struct Piece {
  static constexpr int kN = kBytes / (int)sizeof(T), kWords = kBytes < 4 ? 1 : kBytes / 4;
  static_assert(kN >= 1, "a piece holds an element");
  uint32_t w[kWords];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  __device__ __forceinline__ void load(const T *at) {
    if constexpr (kBytes == 16) {
      const uint4 u = *reinterpret_cast<const uint4 *>(at);
      w[0] = u.x;
      w[1] = u.y;
      w[2] = u.z;
      w[3] = u.w;
    } else if constexpr (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t *>(at);
    } else {
      w[0] = *reinterpret_cast<const uint16_t *>(at);
    }
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
  }
  __device__ __forceinline__ static void store(T *at, const float (&v)[kN]) {
    if constexpr (sizeof(T) == 4) {
      if constexpr (kBytes == 16) *reinterpret_cast<float4 *>(at) = make_float4(v[0], v[1], v[2], v[3]);
      else *at = v[0];
    } else if constexpr (kBytes == 2) {
      *at = __float2bfloat16_rn(v[0]);
    } else {
      uint32_t u[kWords];
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const __nv_bfloat162 both = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t *>(&both);
      }
      if constexpr (kBytes == 16) *reinterpret_cast<uint4 *>(at) = make_uint4(u[0], u[1], u[2], u[3]);
      else *reinterpret_cast<uint32_t *>(at) = u[0];
    }
  }
};

__device__ __forceinline__ void copy_async(void *to, const void *from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// Sums over the threads of a row: `team` of them, a power of two below a warp's 32, or the whole block.
struct RowSum {
  int team;
  float *s;  // of 2 x 32 floats, used by turns
  __device__ __forceinline__ float operator()(float x) {
    if (team < 32) {
      for (int d = team >> 1; d; d >>= 1) x += __shfl_xor_sync(kAll, x, d);
      return x;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(kAll, x, d);
    if (team == 32) return x;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    float sum = 0.0f;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) sum += s[w];
    s = reinterpret_cast<float *>(reinterpret_cast<uintptr_t>(s) ^ 128);
    return sum;
  }
};

// 1 / rms(a).  Squares past fp32 are summed again of values 2^-80 as large, with eps 2^-160 as large.
template <int kP, int kN, typename Value>
__device__ __forceinline__ float unit_of(const Value &value, float eps, int hidden, RowSum &sum) {
  float mine = 0.0f;
  if constexpr (kN > 1) {
    unsigned long long two = 0;
#pragma unroll
    for (int p = 0; p < kP; ++p)
#pragma unroll
      for (int e = 0; e < kN; e += 2) {
        const unsigned long long v = pack_f32x2(value(p, e), value(p, e + 1));
        two = fma_f32x2(v, v, two);
      }
    float odd;
    unpack_f32x2(two, mine, odd);
    mine += odd;
  } else {
#pragma unroll
    for (int p = 0; p < kP; ++p) mine = fmaf(value(p, 0), value(p, 0), mine);
  }
  const float squares = sum(mine);
  const bool fine = squares <= FLT_MAX;
  const float u = rsqrtf(squares / (float)hidden + eps);
  if (__all_sync(kAll, fine)) return u;  // the same in all warps of a row
  const float less = 0x1p-80f;
  mine = 0.0f;
#pragma unroll
  for (int p = 0; p < kP; ++p)
#pragma unroll
    for (int e = 0; e < kN; ++e) mine = fmaf(value(p, e) * less, value(p, e) * less, mine);
  const float again = rsqrtf(sum(mine) / (float)hidden + eps * less * less);
  return fine ? u : less * again;  // 2^-128 at least, which has 21 bits
}

// v = (factor w) v, and to = scale (gate) v + to, of a piece's values.
template <int kN, typename W>
__device__ __forceinline__ void multiply(float (&v)[kN], float factor, const W &w) {
  if constexpr (kN > 1) {
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
      const unsigned long long two = mul_f32x2(mul_f32x2(pack_f32x2(v[e], v[e + 1]), splat_f32x2(factor)), pack_f32x2(w[e], w[e + 1]));
      unpack_f32x2(two, v[e], v[e + 1]);
    }
  } else {
    v[0] = v[0] * factor * w[0];
  }
}
template <int kN, typename W>
__device__ __forceinline__ void add(float (&to)[kN], const float (&v)[kN], float scale, const W *gate) {
  if constexpr (kN > 1) {
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
      const unsigned long long f = gate ? mul_f32x2(splat_f32x2(scale), pack_f32x2((*gate)[e], (*gate)[e + 1])) : splat_f32x2(scale);
      unpack_f32x2(fma_f32x2(f, pack_f32x2(v[e], v[e + 1]), pack_f32x2(to[e], to[e + 1])), to[e], to[e + 1]);
    }
  } else {
    to[0] = fmaf(gate ? scale * (*gate)[0] : scale, v[0], to[0]);
  }
}

// A team of threads for each row, kP pieces of kBytes each; a block has blockDim.x / team rows.  (In bf16 two forms spill: 2 pieces
// of 16 bytes 40 bytes of a thread stored and 12 loaded, 16 pieces of 4 112 and 56.)
template <int kBytes, int kP>
constexpr int kMostThreads = kBytes < 16 && kP <= 4 ? 1024 : 512;
template <typename T, int kBytes, int kP>
__global__ void __launch_bounds__(kMostThreads<kBytes, kP>, kP <= 2 ? 1024 / kMostThreads<kBytes, kP> : 1)
    residual_norm_kernel(NormArgs a, int team) {
  using P = Piece<T, kBytes>;
  constexpr int kN = P::kN;
  __shared__ alignas(256) float s_sum[64];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int rows = blockDim.x / team, mine = rows > 1 ? threadIdx.x % team : threadIdx.x;
  const int64_t row = (int64_t)blockIdx.x * rows + (rows > 1 ? threadIdx.x / team : 0);
  RowSum sum{team, s_sum};
  P x[kP], y[kP], gate[kP];
  const auto at = [&](int p) { return (p * team + mine) * kN; };
  const auto here = [&](int p) { return row < a.n && at(p) < a.hidden; };
#pragma unroll
  for (int p = 0; p < kP; ++p) {
    x[p].clear();
    y[p].clear();
    gate[p].clear();
    if (!here(p)) continue;
    x[p].load((const T *)a.x + row * a.x_row + at(p));
    if (a.y) y[p].load((const T *)a.y + row * a.y_row + at(p));
    if (a.gate) gate[p].load((const T *)a.gate + row * a.gate_row + at(p));
  }
  float s[kP][kN];
#pragma unroll
  for (int p = 0; p < kP; ++p)
#pragma unroll
    for (int e = 0; e < kN; ++e) s[p][e] = x[p][e];
  if (a.y) {
    float u = 1.0f;
    if (a.out_weight) u = unit_of<kP, kN>([&](int p, int e) { return y[p][e]; }, a.eps, a.hidden, sum);
#pragma unroll
    for (int p = 0; p < kP; ++p) {
      if (!here(p)) continue;
      float z[kN];
#pragma unroll
      for (int e = 0; e < kN; ++e) z[e] = y[p][e];
      if (a.out_weight) {
        P w;
        w.load((const T *)a.out_weight + at(p));
        multiply(z, u, w);
      }
      add(s[p], z, a.scale, a.gate ? &gate[p] : nullptr);
      if (a.sum) P::store((T *)a.sum + row * a.sum_row + at(p), s[p]);
    }
  }
  if (!a.normed) return;
  const float u = unit_of<kP, kN>([&](int p, int e) { return s[p][e]; }, a.eps, a.hidden, sum);
#pragma unroll
  for (int p = 0; p < kP; ++p) {
    if (!here(p)) continue;
    P w;
    w.load((const T *)a.weight + at(p));
    multiply(s[p], u, w);
    P::store((T *)a.normed + row * a.normed_row + at(p), s[p]);
  }
}

// The same for more rows than the GPU works on at once: a block takes row after row, and each of its threads has its
// pieces of the next rows on their way to shared memory, where it alone reads them, so that HBM is not left waiting
// while a row's sums are formed: 16,384 rows of 4,096 in 99 us, 105 with a block for each row.
constexpr int kStages = 3;
template <typename T, int kP>
__global__ void __launch_bounds__(512, 2) residual_norm_rows_kernel(NormArgs a) {
  using P = Piece<T, 16>;
  constexpr int kN = P::kN;
  extern __shared__ __align__(16) uint4 s_rows[];  // [stage][x, y, gate][piece][thread]
  __shared__ alignas(256) float s_sum[64];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int threads = blockDim.x, mine = threadIdx.x;
  const bool gates = a.gate && a.gate_row;
  const int arrays = 2 + gates;
  RowSum sum{threads, s_sum};
  const auto at = [&](int p) { return (p * threads + mine) * kN; };
  const auto slot = [&](int stage, int array, int p) { return s_rows + ((stage * arrays + array) * kP + p) * threads + mine; };
  const auto ask = [&](int64_t row, int stage) {
    if (row < a.n)
#pragma unroll
      for (int p = 0; p < kP; ++p) {
        if (at(p) >= a.hidden) continue;
        copy_async(slot(stage, 0, p), (const T *)a.x + row * a.x_row + at(p));
        copy_async(slot(stage, 1, p), (const T *)a.y + row * a.y_row + at(p));
        if (gates) copy_async(slot(stage, 2, p), (const T *)a.gate + row * a.gate_row + at(p));
      }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int i = 0; i < kStages - 1; ++i) ask(blockIdx.x + (int64_t)i * gridDim.x, i);
  int stage = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    ask(row + (int64_t)(kStages - 1) * gridDim.x, stage == 0 ? kStages - 1 : stage - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    P y[kP];
    float s[kP][kN];
#pragma unroll
    for (int p = 0; p < kP; ++p) {
      y[p].clear();
      if (at(p) < a.hidden) y[p].load((const T *)slot(stage, 1, p));
    }
    float u = 1.0f;
    if (a.out_weight) u = unit_of<kP, kN>([&](int p, int e) { return y[p][e]; }, a.eps, a.hidden, sum);
#pragma unroll
    for (int p = 0; p < kP; ++p) {
#pragma unroll
      for (int e = 0; e < kN; ++e) s[p][e] = 0.0f;
      if (at(p) >= a.hidden) continue;
      P x, w, gate;
      x.load((const T *)slot(stage, 0, p));
      if (a.gate) gate.load(gates ? (const T *)slot(stage, 2, p) : (const T *)a.gate + at(p));
      float z[kN];
#pragma unroll
      for (int e = 0; e < kN; ++e) {
        s[p][e] = x[e];
        z[e] = y[p][e];
      }
      if (a.out_weight) {
        w.load((const T *)a.out_weight + at(p));
        multiply(z, u, w);
      }
      add(s[p], z, a.scale, a.gate ? &gate : nullptr);
      if (a.sum) P::store((T *)a.sum + row * a.sum_row + at(p), s[p]);
    }
    if (a.normed) {
      const float v = unit_of<kP, kN>([&](int p, int e) { return s[p][e]; }, a.eps, a.hidden, sum);
#pragma unroll
      for (int p = 0; p < kP; ++p) {
        if (at(p) >= a.hidden) continue;
        P w;
        w.load((const T *)a.weight + at(p));
        multiply(s[p], v, w);
        P::store((T *)a.normed + row * a.normed_row + at(p), s[p]);
      }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
}

// The same for rows that the registers do not hold: x, y and the gate are read again for each of a row's sums,
// from L1 or L2.  Nothing is written before its last read: an element belongs to one thread.
template <typename T, int kBytes>
__global__ void __launch_bounds__(1024) residual_norm_long_kernel(NormArgs a) {
  using P = Piece<T, kBytes>;
  constexpr int kN = P::kN;
  __shared__ alignas(256) float s_sum[64];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t row = blockIdx.x;
  RowSum sum{(int)blockDim.x, s_sum};
  const auto unit = [&](const auto &values) {  // of what values(at, v) puts in v
    float first = 1.0f, v[kN];
    for (;;) {
      float mine = 0.0f;
      for (int at = threadIdx.x * kN; at < a.hidden; at += blockDim.x * kN) {
        values(at, v);
#pragma unroll
        for (int e = 0; e < kN; ++e) mine = fmaf(v[e] * first, v[e] * first, mine);
      }
      const float squares = sum(mine);
      if (first != 1.0f) return first * rsqrtf(squares / (float)a.hidden + a.eps * first * first);
      if (squares <= FLT_MAX) return rsqrtf(squares / (float)a.hidden + a.eps);
      first = 0x1p-80f;
    }
  };
  const auto block = [&](int at, float (&v)[kN]) {
    P y;
    y.load((const T *)a.y + row * a.y_row + at);
#pragma unroll
    for (int e = 0; e < kN; ++e) v[e] = y[e];
  };
  float u = 1.0f;
  if (a.y && a.out_weight) u = unit(block);
  const auto total = [&](int at, float (&v)[kN]) {
    P x, y, w;
    x.load((const T *)a.x + row * a.x_row + at);
    if (!a.y) {
#pragma unroll
      for (int e = 0; e < kN; ++e) v[e] = x[e];
      return;
    }
    block(at, v);
    if (a.out_weight) {
      w.load((const T *)a.out_weight + at);
#pragma unroll
      for (int e = 0; e < kN; ++e) v[e] = v[e] * u * w[e];
    }
    if (a.gate) w.load((const T *)a.gate + row * a.gate_row + at);
#pragma unroll
    for (int e = 0; e < kN; ++e) v[e] = fmaf(a.gate ? a.scale * w[e] : a.scale, v[e], x[e]);
  };
  float whole = 1.0f;
  if (a.normed) whole = unit(total);
  for (int at = threadIdx.x * kN; at < a.hidden; at += blockDim.x * kN) {
    float v[kN];
    total(at, v);
    if (a.sum) P::store((T *)a.sum + row * a.sum_row + at, v);
    if (!a.normed) continue;
    P w;
    w.load((const T *)a.weight + at);
#pragma unroll
    for (int e = 0; e < kN; ++e) v[e] = v[e] * whole * w[e];
    P::store((T *)a.normed + row * a.normed_row + at, v);
  }
}

namespace {

template <typename... Params, typename... Args>
cudaError_t launch_after(unsigned blocks, unsigned threads, int smem, cudaStream_t s, void (*kernel)(Params...), Args... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cfg.stream = s;
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Row after row where blocks take four at least, and a row is work for four warps.
template <typename T>
bool launch_rows(const NormArgs &a, int pieces, cudaStream_t s, cudaError_t *e) {
  constexpr int kP = 2, kMost = kStages * 3 * kP * 512 * 16;
  const int threads = ((pieces - 1) / kP / 32 + 1) * 32, smem = kStages * (2 + (a.gate && a.gate_row)) * kP * threads * 16;
  const int by_smem = 228 * 1024 / (smem + 1280), by_threads = 1024 / threads, blocks = 152 * (by_smem < by_threads ? by_smem : by_threads);
  if (!a.y || pieces <= 128 || pieces > kP * 512 || a.n < 4 * blocks) return false;
  *e = allow_smem((const void *)residual_norm_rows_kernel<T, kP>, smem + (int)sizeof(float) * 64, kMost);
  if (*e == cudaSuccess) *e = launch_after(blocks, threads, smem, s, residual_norm_rows_kernel<T, kP>, a);
  return true;
}

// kP pieces for each thread of a team: a part of a warp or a warp of a block of 256, or a block.
template <typename T, int kBytes, int kP>
cudaError_t launch(const NormArgs &a, int pieces, cudaStream_t s) {
  int team = 1;
  while (team < 32 && team * kP < pieces) team <<= 1;
  if (team * kP < pieces) team = ((pieces - 1) / kP / 32 + 1) * 32;
  const int threads = team <= 32 ? 256 : team, rows = threads / team;
  return launch_after((unsigned)((a.n - 1) / rows + 1), threads, 0, s, residual_norm_kernel<T, kBytes, kP>, a, team);
}

template <typename T, int kBytes>
cudaError_t by_width(const NormArgs &a, cudaStream_t s) {
  constexpr int kN = kBytes / (int)sizeof(T);
  const int pieces = (a.hidden - 1) / kN + 1;
  if (pieces <= 32) return launch<T, kBytes, 1>(a, pieces, s);
  if constexpr (kBytes == 16) {
    cudaError_t e;
    if (launch_rows<T>(a, pieces, s, &e)) return e;
  }
  if (pieces <= 2 * 512) return launch<T, kBytes, 2>(a, pieces, s);
  if (pieces <= 4 * kMostThreads<kBytes, 4>) return launch<T, kBytes, 4>(a, pieces, s);
  if constexpr (kBytes < 16)
    if (pieces <= 16 * 512) return launch<T, kBytes, 16>(a, pieces, s);
  return launch_after((unsigned)a.n, 1024, 0, s, residual_norm_long_kernel<T, kBytes>, a);
}

}  // namespace

cudaError_t launch_residual_norm(int dtype, const NormArgs &a, cudaStream_t s) {
  if (a.n == 0) return cudaSuccess;
  const int size = dtype == COPES_BF16 ? 2 : 4;
  // what every row of every array is aligned to
  uint64_t all = (uint64_t)a.hidden * size;
  const auto array = [&](const void *p, int64_t row) {
    if (p) all |= (uint64_t)(uintptr_t)p | (uint64_t)row * size;
  };
  array(a.x, a.x_row);
  array(a.y, a.y_row);
  array(a.gate, a.gate_row);
  array(a.out_weight, 0);
  array(a.weight, 0);
  array(a.sum, a.sum_row);
  array(a.normed, a.normed_row);
  if (dtype == COPES_BF16) {
    if (all % 16 == 0) return by_width<__nv_bfloat16, 16>(a, s);
    if (all % 4 == 0) return by_width<__nv_bfloat16, 4>(a, s);
    return by_width<__nv_bfloat16, 2>(a, s);
  }
  return all % 16 == 0 ? by_width<float, 16>(a, s) : by_width<float, 4>(a, s);
}

}  // namespace copes
