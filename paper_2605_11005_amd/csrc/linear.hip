// A linear layer, grouped by expert or dense:
//     z = x W[e] + b[e]        y = act(z) + residual
//     dz = dy act'(z)          dx = dz W[e]^T        dW[e] (+)= x^T dz        db[e] (+)= sum_rows dz
// The products are those of expert_bf16.hip and expert_f32.hip; here are what surrounds them, dz with the sums of its columns, and which
// kernel a call takes.
#include "activation.h"
#include "common.h"
#include "kernels.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int SETUP_WORDS = 64;            // ticket counters, then the row offsets of a dense call
__global__ void linear_setup(int32_t* words, int rows) {
  const int i = threadIdx.x;
  if (i < SETUP_WORDS + 2) words[i] = i == SETUP_WORDS + 1 ? rows : 0;
}

template <typename T> constexpr int VEC = 16 / sizeof(T);
__device__ __forceinline__ void values(u32x4 w, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) { v[2 * j] = bf16lo(w[j]); v[2 * j + 1] = bf16hi(w[j]); }
}
__device__ __forceinline__ void values(u32x4 w, float (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ u32x4 words(const float (&v)[8]) {
  return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ u32x4 words(const float (&v)[4]) {
  return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
}

// dz = dy act'(z), rounded to the type that the products take, and the column sums of what it was before, over 64 rows of an expert by
// 64 lanes' 16 bytes.  Four wavefronts take every fourth row each; their sums meet in ascending order.  HBM bound: dy and z in, dz out.
// The sums of row tile i of expert e go to line offsets[e] / 64 + e + i: lines of different tiles differ, as floor((o + n) / 64) + 1 >=
// floor(o / 64) + ceil(n / 64).
constexpr int SUM_ROWS = 64, GRAD_WAVES = 4;
inline long long sum_lines(int rows, int e_cnt) { return rows / SUM_ROWS + (long long)e_cnt; }
template <typename T>
__global__ __launch_bounds__(GRAD_WAVES * WAVE) void act_grad(const int32_t* __restrict__ off, int e_cnt, int N, int act, const T* __restrict__ dy,
                                                              const T* __restrict__ z, T* __restrict__ dz, float* __restrict__ sums) {
  constexpr int V = VEC<T>, WIDTH = WAVE * V;
  __shared__ float part[GRAD_WAVES][V][WAVE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int e, row_tile, col_tile;
  if (!RaggedTiles<SUM_ROWS>(off, e_cnt, lane).tile((N + WIDTH - 1) / WIDTH, blockIdx.x, e, row_tile, col_tile)) return;
  const int first = off[e], row0 = first + row_tile * SUM_ROWS, end = min(off[e + 1], row0 + SUM_ROWS);
  const int c = col_tile * WIDTH + lane * V;
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.f;
  if (c < N)
    with_activation(act, [&](auto a) {
      constexpr int ACT = decltype(a)::value;
#pragma unroll 4
      for (int row = row0 + wave; row < end; row += GRAD_WAVES) {
        const size_t at = (size_t)row * N + c;
        float g[V];
        values(*reinterpret_cast<const u32x4*>(dy + at), g);
        if constexpr (ACT != MOE_ACT_NONE) {
          float v[V];
          values(*reinterpret_cast<const u32x4*>(z + at), v);
#pragma unroll
          for (int j = 0; j < V; ++j) g[j] = act_slope<ACT, sizeof(T) == 2>(v[j], g[j]);
          *reinterpret_cast<u32x4*>(dz + at) = words(g);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += g[j];
      }
    });
  if (!sums) return;
#pragma unroll
  for (int j = 0; j < V; ++j) part[wave][j][lane] = sum[j];
  __syncthreads();
  if (wave || c >= N) return;
  float* const out = sums + ((size_t)(first / SUM_ROWS) + e + row_tile) * N + c;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < GRAD_WAVES; ++w) t += part[w][j][lane];
    out[j] = t;
  }
}

// db of expert blockIdx.y from the sums of its row tiles, in ascending order: wavefront w of 16 adds the w-th part of them, 64 columns a block.
constexpr int BIAS_WAVES = 16;
template <typename T>
__global__ __launch_bounds__(BIAS_WAVES * WAVE) void bias_grad(const int32_t* __restrict__ off, int N, const float* __restrict__ sums, int accumulate,
                                                               T* __restrict__ db) {
  __shared__ float part[BIAS_WAVES][WAVE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * WAVE + lane, e = blockIdx.y;
  const int first = off[e], tiles = (off[e + 1] - first + SUM_ROWS - 1) / SUM_ROWS;
  const int share = (tiles + BIAS_WAVES - 1) / BIAS_WAVES, end = min(tiles, (wave + 1) * share);
  const float* const line = sums + ((size_t)(first / SUM_ROWS) + e) * N;
  float s = 0.f;
  if (c < N)
#pragma unroll 8
    for (int i = wave * share; i < end; ++i) s += line[(size_t)i * N + c];
  part[wave][lane] = s;
  __syncthreads();
  if (wave || c >= N) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < BIAS_WAVES; ++w) s += part[w][lane];
  T* const to = db + (size_t)e * N + c;
  if constexpr (sizeof(T) == 2) *to = (bf16_t)pack_bf16x2(accumulate ? bf16_to_f32(*to) + s : s, 0.f);      // (the hardware's conversion keeps every NaN)
  else *to = accumulate ? *to + s : s;
}

template <typename T>
int gradients(const LinearArgs& l, const int32_t* off, const void* dy, void* dz, void* db, float* sums, int accumulate, hipStream_t s) {
  constexpr int WIDTH = WAVE * VEC<T>;
  if (l.rows > 0) {
    ProfScope prof(MOE_K_LINEAR_ACT, s);
    const long long tiles = ((long long)(l.rows + SUM_ROWS - 1) / SUM_ROWS + l.e_cnt) * ((l.N + WIDTH - 1) / WIDTH);
    hipLaunchKernelGGL(act_grad<T>, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(GRAD_WAVES * WAVE), 0, s, off, l.e_cnt, l.N, l.act, (const T*)dy,
                       (const T*)l.z, (T*)dz, db ? sums : nullptr);
    HIP_CHECK_LAUNCH();
  }
  if (db) {
    ProfScope prof(MOE_K_LINEAR_BIAS, s);
    hipLaunchKernelGGL(bias_grad<T>, dim3((l.N + WAVE - 1) / WAVE, l.e_cnt), dim3(BIAS_WAVES * WAVE), 0, s, off, l.N, sums, accumulate, (T*)db);
    HIP_CHECK_LAUNCH();
  }
  return MOE_OK;
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
constexpr size_t SETUP_BYTES = 512;
static_assert((SETUP_WORDS + 2) * 4 <= SETUP_BYTES, "");
// The backward's workspace: what linear_setup writes, dz, the column sums, then what the products of bf16 take
struct BwdSpace {
  size_t dz, sums, products, end;
  BwdSpace(int dtype, int rows, int K, int N, int e_cnt) {
    dz = SETUP_BYTES;
    sums = dz + align256((size_t)rows * N * (dtype == MOE_BF16 ? 2 : 4));
    products = sums + align256((size_t)sum_lines(rows, e_cnt) * N * 4);
    end = products + (dtype == MOE_BF16 ? MOE_MAX_LOCAL * 4 + linear_split_bytes(K, N) : 0);
  }
};

}  // namespace

size_t linear_fwd_ws_bytes(int dtype, int rows, int K, int N, int e_cnt) { return SETUP_BYTES; }
size_t linear_bwd_ws_bytes(int dtype, int rows, int K, int N, int e_cnt) { return BwdSpace(dtype, rows, K, N, e_cnt).end; }

int launch_linear_fwd(const LinearArgs& l, void* ws, hipStream_t s) {
  if (l.rows == 0 || l.e_cnt == 0) return MOE_OK;
  int32_t* const setup = (int32_t*)ws;
  if (l.dtype == MOE_BF16 || !l.offsets) {
    hipLaunchKernelGGL(linear_setup, dim3(1), dim3(128), 0, s, setup, l.rows);
    HIP_CHECK_LAUNCH();
  }
  if (l.dtype == MOE_BF16) return launch_linear_fwd_tiles(l, setup, s);
  LinearArgs with_offsets = l;
  if (!l.offsets) with_offsets.offsets = setup + SETUP_WORDS;
  return launch_linear_fwd_f32(with_offsets, s);
}

int launch_linear_bwd(const LinearArgs& l, const void* dy, void* dx, void* dw, void* db, int accumulate, void* ws, hipStream_t s) {
  if (l.e_cnt == 0) return MOE_OK;
  const BwdSpace space(l.dtype, l.rows, l.K, l.N, l.e_cnt);
  char* const base = (char*)ws;
  int32_t* const setup = (int32_t*)ws;
  hipLaunchKernelGGL(linear_setup, dim3(1), dim3(128), 0, s, setup, l.rows);
  HIP_CHECK_LAUNCH();
  const int32_t* const off = l.offsets ? l.offsets : setup + SETUP_WORDS;
  const bool through = l.act != MOE_ACT_NONE;
  void* const dz = through ? base + space.dz : nullptr;
  int rc;
  if (db || (through && (dx || dw))) {
    float* const sums = (float*)(base + space.sums);
    rc = l.dtype == MOE_BF16 ? gradients<bf16_t>(l, off, dy, dz, db, sums, accumulate, s) : gradients<float>(l, off, dy, dz, db, sums, accumulate, s);
    if (rc) return rc;
  }
  const void* const g = through ? dz : dy;
  if (l.dtype == MOE_BF16) return launch_linear_bwd_tiles(l, g, dx, dw, accumulate, setup, base + space.products, s);
  LinearArgs with_offsets = l;
  with_offsets.offsets = off;
  return launch_linear_bwd_f32(with_offsets, g, dx, dw, accumulate, s);
}
