// The gradient of the linear layer's biases: of every expert the sums of its row tiles, in ascending order, 64 columns a block of 256 threads.
#pragma once
#include "common.h"
#include "linear.h"

namespace {

constexpr int BIAS_THREADS = 256;
inline unsigned bias_blocks(int N, int e_cnt) { return (unsigned)e_cnt * ((N + WAVE - 1) / WAVE); }

// wavefront w of four adds the w-th quarter of the tiles
template <typename T>
__device__ __forceinline__ void bias_columns(const BiasGrad& p, int block, float* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cols = (p.N + WAVE - 1) / WAVE, e = block / cols, c = (block - e * cols) * WAVE + lane;
  const int first = p.off ? p.off[e] : 0, tiles = ((p.off ? p.off[e + 1] : p.rows) - first + LINEAR_SUM_ROWS - 1) / LINEAR_SUM_ROWS;
  const int share = (tiles + 3) / 4, end = min(tiles, (wave + 1) * share);
  const float* const line = p.sums + ((size_t)(first / LINEAR_SUM_ROWS) + e) * p.N;
  float s = 0.f;
  if (c < p.N)
#pragma unroll 8
    for (int i = wave * share; i < end; ++i) s += line[(size_t)i * p.N + c];
  part[threadIdx.x] = s;
  __syncthreads();
  if (wave || c >= p.N) return;
  s = ((part[lane] + part[64 + lane]) + part[128 + lane]) + part[192 + lane];
  T* const to = (T*)p.db + (size_t)e * p.N + c;
  if constexpr (sizeof(T) == 2) *to = (bf16_t)pack_bf16x2(p.accumulate ? bf16_to_f32(*to) + s : s, 0.f);      // (the hardware's conversion keeps every NaN)
  else *to = p.accumulate ? *to + s : s;
}

}  // namespace
