// What the kernels that keep a row in the registers of its threads share: vectors of 16 bytes per lane, sums over a row, and the
// sums over the rows of what its blocks leave.
#pragma once
#include "common.h"
#include "kernels.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T> constexpr int VEC = 16 / sizeof(T);

// N elements as they lie in memory, and as floats
template <typename T, int N>
struct Raw {
  u32x4 w[N * sizeof(T) / 16];
  template <bool STREAM = false>      // not used again
  __device__ __forceinline__ void load(const T* p, size_t i) {
#pragma unroll
    for (int j = 0; j < (int)(N * sizeof(T) / 16); ++j) {
      const u32x4* const from = reinterpret_cast<const u32x4*>(p + i + j * VEC<T>);
      w[j] = STREAM ? __builtin_nontemporal_load(from) : *from;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < (int)(N * sizeof(T) / 16); ++j) w[j] = 0;
  }
  __device__ __forceinline__ void values(float (&v)[N]) const {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (sizeof(T) == 4) v[j] = __uint_as_float(w[j / 4][j % 4]);
      else v[j] = j % 2 ? bf16hi(w[j / 8][j % 8 / 2]) : bf16lo(w[j / 8][j % 8 / 2]);
    }
  }
};
template <int N, bool STREAM = false, typename T>
__device__ __forceinline__ void unpack(const T* p, size_t i, float (&v)[N]) {
  Raw<T, N> raw;
  raw.template load<STREAM>(p, i);
  raw.values(v);
}
template <bool STREAM>
__device__ __forceinline__ void store_words(void* p, u32x4 w) {
  if constexpr (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = w;
}
template <int N, bool STREAM = false>
__device__ __forceinline__ void pack(bf16_t* p, size_t i, const float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N / 8; ++j) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = pack_bf16x2(v[8 * j + 2 * k], v[8 * j + 2 * k + 1]);
    store_words<STREAM>(p + i + 8 * j, w);
  }
}
template <int N, bool STREAM = false>
__device__ __forceinline__ void pack(float* p, size_t i, const float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __float_as_uint(v[4 * j + k]);
    store_words<STREAM>(p + i + 4 * j, w);
  }
}

__device__ __forceinline__ float wave_total(float v) {
#pragma unroll
  for (int m = 1; m < WAVE; m *= 2) v += __shfl_xor(v, m);
  return v;
}
constexpr int MOST_WAVES = 16;
// Sums over a row's threads: its wavefronts' sums meet in LDS, in their order.  Two places in turn: a place is written again only after the
// barrier of the sum in between, which every wavefront passes when it has read the place.
struct RowSum {
  float (*red)[MOST_WAVES];
  int waves, turn = 0;
  __device__ __forceinline__ float operator()(float v) {
    v = wave_total(v);
    if (waves == 1) return v;
    float* const place = red[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) place[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
    for (int w = 0; w < waves; ++w) s += place[w];
    return s;
  }
};

// The blocks' column sums in ascending order: wavefront w of 16 adds the w-th part of them, 64 columns a block.
constexpr int SUM_WAVES = 16;
template <typename T>
__global__ __launch_bounds__(SUM_WAVES * WAVE) void column_sums(const float* __restrict__ sums, int blocks, int d, int accumulate, T* __restrict__ out0,
                                                                T* __restrict__ out1) {
  __shared__ float part[SUM_WAVES][WAVE];
  T* const out = blockIdx.y ? out1 : out0;
  if (!out) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * WAVE + lane;
  const int share = (blocks + SUM_WAVES - 1) / SUM_WAVES, end = min(blocks, (wave + 1) * share);
  float s = 0.f;
  if (c < d)
#pragma unroll 8
    for (int b = wave * share; b < end; ++b) s += sums[((size_t)b * 2 + blockIdx.y) * d + c];
  part[wave][lane] = s;
  __syncthreads();
  if (wave || c >= d) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < SUM_WAVES; ++w) s += part[w][lane];
  // (the hardware's conversion: a sum may be NaN of any payload, from the residual stream or the gate)
  if constexpr (sizeof(T) == 2) out[c] = (bf16_t)pack_bf16x2(accumulate ? bf16_to_f32(out[c]) + s : s, 0.f);
  else out[c] = accumulate ? out[c] + s : s;
}

// threads of a row at `steps` vectors each, whole wavefronts
inline int row_threads(int vecs, int steps) { return WAVE * ((vecs + WAVE * steps - 1) / (WAVE * steps)); }

template <typename F>
int by_types(int dtype, int res_dtype, F f) {
  if (dtype == MOE_F32) return f((float*)nullptr, (float*)nullptr);
  if (res_dtype == MOE_F32) return f((bf16_t*)nullptr, (float*)nullptr);
  return f((bf16_t*)nullptr, (bf16_t*)nullptr);
}

}  // namespace
