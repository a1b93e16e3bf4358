// The gradient of the linear layer's biases: of every expert the sums of its row tiles, in ascending order, or of few rows themselves, 64 columns a block of 256 threads.
#pragma once
#include "common.h"
#include "linear_finish.h"

namespace {

constexpr int BIAS_THREADS = 256;
inline unsigned bias_blocks(int N, int e_cnt) { return (unsigned)e_cnt * ((N + WAVE - 1) / WAVE); }

// wavefront w of four adds the w-th quarter of the tiles, or every fourth load of rows
template <typename T>
__device__ __forceinline__ void bias_columns(const BiasGrad& p, int block, float* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cols = (p.N + WAVE - 1) / WAVE, e = block / cols, c = (block - e * cols) * WAVE + lane;
  const int first = p.off ? p.off[e] : 0, end_row = p.off ? p.off[e + 1] : p.rows;
  float s = 0.f;
  if (p.dy) {
    constexpr int N = 16 / sizeof(T), LANES = WAVE / N, AT_ONCE = WAVE / LANES;      // lanes and rows of a wavefront's load of 64 columns
    const int col = c - lane + lane % LANES * N;
    float v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = 0.f;
    if (col < p.N)
      with_activation(p.act, [&](auto a) {
        constexpr int ACT = decltype(a)::value;
#pragma unroll 4
        for (int row = first + wave * AT_ONCE + lane / LANES; row < end_row; row += 4 * AT_ONCE) {
          const size_t at = (size_t)row * p.N + col;
          float g[N];
          values(*reinterpret_cast<const u32x4*>((const T*)p.dy + at), g);
          if constexpr (ACT != MOE_ACT_NONE) {
            float z[N];
            values(*reinterpret_cast<const u32x4*>((const T*)p.z + at), z);
#pragma unroll
            for (int j = 0; j < N; ++j) g[j] = act_slope<ACT, sizeof(T) == 2>(z[j], g[j]);
          }
#pragma unroll
          for (int j = 0; j < N; ++j) v[j] += g[j];
        }
      });
#pragma unroll
    for (int j = 0; j < N; ++j) {
#pragma unroll
      for (int m = LANES; m < WAVE; m *= 2) v[j] += __shfl_xor(v[j], m);
      const float mine = __shfl(v[j], lane / N);           // column c is element lane % N of lane lane / N
      s = lane % N == j ? mine : s;
    }
  } else {
    const int tiles = (end_row - first + LINEAR_SUM_ROWS - 1) / LINEAR_SUM_ROWS, share = (tiles + 3) / 4, end = min(tiles, (wave + 1) * share);
    const float* const line = p.sums + ((size_t)(first / LINEAR_SUM_ROWS) + e) * p.N;
    if (c < p.N)
#pragma unroll 8
      for (int i = wave * share; i < end; ++i) s += line[(size_t)i * p.N + c];
  }
  part[threadIdx.x] = s;
  __syncthreads();
  if (wave || c >= p.N) return;
  s = ((part[lane] + part[64 + lane]) + part[128 + lane]) + part[192 + lane];
  T* const to = (T*)p.db + (size_t)e * p.N + c;
  if constexpr (sizeof(T) == 2) *to = (bf16_t)pack_bf16x2(p.accumulate ? bf16_to_f32(*to) + s : s, 0.f);      // (the hardware's conversion keeps every NaN)
  else *to = p.accumulate ? *to + s : s;
}

}  // namespace
