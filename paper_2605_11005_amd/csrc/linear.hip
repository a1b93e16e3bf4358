// A linear layer, grouped by expert or dense:
//     z = x W[e] + b[e]        y = act(z) + residual
//     dz = dy act'(z)          dx (+)= dz W[e]^T     dW[e] (+)= x^T dz        db[e] (+)= sum_rows dz
// The products are those of linear_few.hip, linear_tiles.hip and, where they fill the chip, expert_bf16.hip, in fp32 of expert_f32.hip; here are what
// surrounds them, dz with the sums of its columns, and which kernel a call takes.
#include "activation.h"
#include "bias_grad.h"
#include "common.h"
#include "linear_finish.h"

namespace {

constexpr int SETUP_WORDS = 64;            // ticket counters of the large tiles
__device__ __forceinline__ void clear(int32_t* words) {
  if (threadIdx.x < SETUP_WORDS) words[threadIdx.x] = 0;
}
__global__ void linear_setup(int32_t* words) { clear(words); }

// dz = dy act'(z), rounded to the type that the products take, and the column sums of what it was before, over 64 rows of an expert by
// 64 lanes' 16 bytes.  Eight wavefronts take every eighth row each; their sums meet in ascending order.  HBM bound: dy and z in, dz out.
// (The bf16 matrix instruction takes both operands in bf16, and dz's rest as a second operand would double both products.  Behind an activation dx and dw
// are then off by 2.35e-3 of their root mean square, where the rounding of their own values takes 1.66e-3: 16384 rows of 7168 to 2048, gelu, against
// 64 bits.  Without one dz is dy, and nothing is rounded.)
// STREAM: with an activation neither dy nor z is read again, and dz is.  Where they take half of the Infinity Cache and more, loads that leave no trace
// there bring a whole backward of 16384 rows of 256 to 4096 from 176 to 158 us, of 2048 to 7168 from 952 to 926; tensors that lie in the cache already are
// not kept by them: 4096 rows of 1024 to 4096 101 -> 93 us from memory, but 90 -> 93 in a loop over the same ones.
// The sums of row tile i of expert e go to line offsets[e] / 64 + e + i: lines of different tiles differ, as floor((o + n) / 64) + 1 >=
// floor(o / 64) + ceil(n / 64).
constexpr int SUM_ROWS = LINEAR_SUM_ROWS, GRAD_WAVES = 8;
inline long long sum_lines(int rows, int e_cnt) { return rows / SUM_ROWS + (long long)e_cnt; }
template <typename T, bool STREAM>
__global__ __launch_bounds__(GRAD_WAVES * WAVE) void act_grad(const int32_t* __restrict__ off, int rows, int e_cnt, int N, int act,
                                                              const T* __restrict__ dy, const T* __restrict__ z, T* __restrict__ dz,
                                                              float* __restrict__ sums, int32_t* __restrict__ setup) {
  if (setup && blockIdx.x == 0) clear(setup);
  constexpr int V = VEC<T>, WIDTH = WAVE * V;
  __shared__ float part[GRAD_WAVES][V][WAVE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int cols = (N + WIDTH - 1) / WIDTH;
  int e = 0, row_tile = blockIdx.x / cols, col_tile = blockIdx.x % cols, first = 0;
  if (off) {
    if (!RaggedTiles<SUM_ROWS>(off, e_cnt, lane).tile(cols, blockIdx.x, e, row_tile, col_tile)) return;
    first = off[e];
    rows = off[e + 1];
  }
  const int row0 = first + row_tile * SUM_ROWS, end = min(rows, row0 + SUM_ROWS);
  if (row0 >= end) return;
  const int c = col_tile * WIDTH + lane * V;
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.f;
  if (c < N)
    with_activation(act, [&](auto a) {
      constexpr int ACT = decltype(a)::value;
#pragma unroll 8
      for (int row = row0 + wave; row < end; row += GRAD_WAVES) {
        const size_t at = (size_t)row * N + c;
        float g[V];
        const u32x4* const from = reinterpret_cast<const u32x4*>(dy + at);
        values(STREAM ? __builtin_nontemporal_load(from) : *from, g);
        if constexpr (ACT != MOE_ACT_NONE) {
          float v[V];
          const u32x4* const of = reinterpret_cast<const u32x4*>(z + at);
          values(STREAM ? __builtin_nontemporal_load(of) : *of, v);
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

// dz alone, 16 bytes a thread, for few rows, whose sums the products' launch forms by itself
constexpr int DZ_THREADS = 256;
template <typename T>
__global__ __launch_bounds__(DZ_THREADS) void act_grad_few(const int32_t* __restrict__ off, int rows, int e_cnt, int N, int act,
                                                           const T* __restrict__ dy, const T* __restrict__ z, T* __restrict__ dz) {
  constexpr int V = VEC<T>;
  const size_t at = ((size_t)blockIdx.x * DZ_THREADS + threadIdx.x) * V;
  if (at >= (size_t)(off ? off[e_cnt] : rows) * N) return;
  float g[V], v[V];
  values(*reinterpret_cast<const u32x4*>(dy + at), g);
  values(*reinterpret_cast<const u32x4*>(z + at), v);
  with_activation(act, [&](auto a) {
#pragma unroll
    for (int j = 0; j < V; ++j) g[j] = act_slope<decltype(a)::value, sizeof(T) == 2>(v[j], g[j]);
  });
  *reinterpret_cast<u32x4*>(dz + at) = words(g);
}

// db, where no launch of the products takes it along
__global__ __launch_bounds__(BIAS_THREADS) void bias_grad(BiasGrad p) {
  __shared__ float part[BIAS_THREADS];
  bias_columns<bf16_t>(p, blockIdx.x, part);
}

// few: sums by the launch behind
template <typename T>
int gradients(const LinearArgs& l, const void* dy, void* dz, float* sums, bool few, int32_t* setup, hipStream_t s) {
  constexpr int WIDTH = WAVE * VEC<T>;
  ProfScope prof(MOE_K_LINEAR_ACT, s);
  if (few) {
    const long long n = (long long)l.rows * l.N / VEC<T>;
    hipLaunchKernelGGL(act_grad_few<T>, dim3((unsigned)((n + DZ_THREADS - 1) / DZ_THREADS)), dim3(DZ_THREADS), 0, s, l.offsets, l.rows, l.e_cnt, l.N, l.act,
                       (const T*)dy, (const T*)l.z, (T*)dz);
    HIP_CHECK_LAUNCH();
  } else {
    const long long tiles = ((long long)(l.rows + SUM_ROWS - 1) / SUM_ROWS + l.e_cnt) * ((l.N + WIDTH - 1) / WIDTH);
    const bool stream = l.act != MOE_ACT_NONE && 2.0 * l.rows * l.N * sizeof(T) >= (double)(128ll << 20);
    const auto kernel = stream ? act_grad<T, true> : act_grad<T, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(GRAD_WAVES * WAVE), 0, s, l.offsets, l.rows, l.e_cnt, l.N, l.act, (const T*)dy,
                       (const T*)l.z, (T*)dz, sums, setup);
    HIP_CHECK_LAUNCH();
  }
  return MOE_OK;
}

enum Route { FEW_ROWS, TILES, LARGE };
// Time in us of the 256x256 tiles, with all experts alike: whole rounds of the chip, each tile by the length of its contraction
struct Large {
  long long n;             // tiles
  float each;
};
inline long long tiles256(int n) { return (n + 255) / 256; }
inline Large large_rows(const LinearArgs& l, int N, int K) {
  const long long per = (l.rows + l.e_cnt - 1) / l.e_cnt;
  return {l.e_cnt * tiles256((int)per) * tiles256(N), 0.026f * (float)K + 3.f};
}
inline float large_fwd_time(const LinearArgs& l) {
  const Large f = large_rows(l, l.N, l.K);
  return 10.f + (float)((f.n + 255) / 256) * f.each;
}
// dx's tiles first, dW's after them by whoever is free: CUs that ran a last tile of dx, and the others
inline float large_bwd_time(const LinearArgs& l, bool dx, bool dw) {
  const Large x = dx ? large_rows(l, l.K, l.N) : Large{0, 0.f};
  const long long per = (l.rows + l.e_cnt - 1) / l.e_cnt;
  const float each = 0.027f * (float)per + 6.f;
  long long left = dw ? l.e_cnt * tiles256(l.K) * tiles256(l.N) : 0;
  const long long late = x.n % 256, early = 256 - late;
  float at_early = (float)(x.n / 256) * x.each, at_late = at_early + (late ? x.each : 0.f);
  if (left > 16384) {                                // (many rounds: everybody ends together)
    const float mean = ((float)early * at_early + (float)late * at_late) / 256.f;
    at_early = at_late = mean + (float)(left / 256) * each;
    left %= 256;
  }
  while (left > 0) {
    const bool e = at_early <= at_late || !late;
    left -= e ? early : late;
    (e ? at_early : at_late) += each;
  }
  return 15.f + (at_early > at_late ? at_early : at_late);
}
// Forward, us.  Few rows' kernel / 128x128 tiles: 16 rows of 4096 to 4096 12.4 / 14.2, 32 rows 13.4 / 14.5 (of 14336 to 4096 33.2 / 30.7), 64 rows 16.2 / 16.4 and
// 39.8 / 32.7; 16 experts of 2880 to 2880 with 24 rows each 57.6 / 58.9, 40 62.8 / 61.4, 64 68.9 / 63.4.  128x128 / 256x256: 4096 rows of 2880 to 2880
// 85 / 87, of 4096 to 4096 145 / 127, of 4096 to 1536 59 / 82, 8192 of those 124 / 114; 16 experts' 256 rows of 2880 to 2880 104 / 96, 1024 rows 328 / 278.
// Backward: 4096 rows of 2880 to 2880 165 / 206, of 4096 to 4096 295 / 266, of 7168 to 2048 268 / 252; 16 experts' 1024 rows of 2880 690 / 632.
Route forward_route(const LinearArgs& l) {
  if (l.rows <= 32ll * l.e_cnt) return FEW_ROWS;
  return linear_tiles_fwd_time(l) <= large_fwd_time(l) ? TILES : LARGE;
}
Route backward_route(const LinearArgs& l, bool dx, bool dw) {
  return linear_tiles_bwd_time(l, dx, dw) <= large_bwd_time(l, dx, dw) ? TILES : LARGE;
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
constexpr size_t SETUP_BYTES = SETUP_WORDS * 4;
// The backward's workspace: the ticket counters, dz, the column sums, then what the products take
struct BwdSpace {
  size_t dz, sums, products, dw_parts, end;
  BwdSpace(int dtype, int rows, int K, int N, int e_cnt) {
    dz = SETUP_BYTES;
    sums = dz + align256((size_t)rows * N * (dtype == MOE_BF16 ? 2 : 4));
    products = sums + align256((size_t)sum_lines(rows, e_cnt) * N * 4);
    const auto parts = dtype == MOE_BF16 ? linear_parts_bytes : linear_f32_parts_bytes;
    dw_parts = products + align256(parts(rows, K));
    end = dw_parts + parts((long long)e_cnt * K, N);
    const size_t pieces = products + (dtype == MOE_BF16 ? MOE_MAX_LOCAL * 4 + linear_split_bytes(K, N) : 0);
    if (end < pieces) end = pieces;
  }
};

}  // namespace

size_t linear_fwd_ws_bytes(int dtype, int rows, int K, int N, int e_cnt) {
  if (dtype != MOE_BF16) return SETUP_BYTES + linear_f32_parts_bytes(rows, N);
  const size_t few = linear_few_ws_bytes(rows, N), parts = linear_parts_bytes(rows, N);
  return SETUP_BYTES + (few > parts ? few : parts);
}
size_t linear_bwd_ws_bytes(int dtype, int rows, int K, int N, int e_cnt) { return BwdSpace(dtype, rows, K, N, e_cnt).end; }

int launch_linear_fwd(const LinearArgs& l, void* ws, hipStream_t s) {
  if (l.rows == 0 || l.e_cnt == 0) return MOE_OK;
  void* const parts = (char*)ws + SETUP_BYTES;
  if (l.dtype == MOE_F32) return launch_linear_fwd_f32(l, parts, s);
  const Route route = forward_route(l);
  if (route == FEW_ROWS) return launch_linear_few(l, parts, s);
  if (route == TILES) return launch_linear_tiles_fwd(l, parts, s);
  hipLaunchKernelGGL(linear_setup, dim3(1), dim3(SETUP_WORDS), 0, s, (int32_t*)ws);
  HIP_CHECK_LAUNCH();
  return launch_linear_fwd_large(l, (int32_t*)ws, s);
}

int launch_linear_bwd(const LinearArgs& l, const void* dy, void* dx, int dx_accumulate, void* dw, void* db, int accumulate, void* ws, hipStream_t s) {
  if (l.e_cnt == 0) return MOE_OK;
  const BwdSpace space(l.dtype, l.rows, l.K, l.N, l.e_cnt);
  char* const base = (char*)ws;
  const bool through = l.act != MOE_ACT_NONE, bf16 = l.dtype == MOE_BF16, large = bf16 && backward_route(l, dx, dw) == LARGE;
  void* const dz = through ? base + space.dz : nullptr;
  float* const sums = (float*)(base + space.sums);
  int32_t* const setup = large ? (int32_t*)ws : nullptr;
  int rc;
  // Few rows: the products' launch sums dy act'(z) by itself, so that without an activation there is no launch in front of it, and with one a short one.
  // fp32's dz is not rounded: its columns are what db sums.  us, sums in front / so, gelu: bf16 200 rows of 1024 to 1024 22.7 / 15.7, 500 rows 25 / 19, 800
  // rows 28 / 24, 1000 rows 29 / 30, of 520 to 776 27 / 34, 800 rows of 64 to 72 20 / 30; fp32 1000 rows of 1024 to 1024 53 / 47, of 520 to 776 41 / 32.
  const bool few = !large && l.rows <= (bf16 ? 640 : 1024), of_dz = !bf16 && through && (dx || dw);
  if (l.rows > 0 && ((db && !few) || (through && (dx || dw)))) {
    rc = bf16 ? gradients<bf16_t>(l, dy, dz, db ? sums : nullptr, few, setup, s) : gradients<float>(l, dy, dz, db ? sums : nullptr, few, setup, s);
    if (rc) return rc;
  } else if (large) {
    hipLaunchKernelGGL(linear_setup, dim3(1), dim3(SETUP_WORDS), 0, s, setup);
    HIP_CHECK_LAUNCH();
  }
  const void* const g = through ? dz : dy;
  const BiasGrad bias = {l.offsets, l.rows, l.N, accumulate, sums, !few ? nullptr : of_dz ? dz : dy, l.z, of_dz ? MOE_ACT_NONE : l.act, db};
  if (!bf16) return launch_linear_bwd_f32(l, g, dx, dx_accumulate, dw, accumulate, bias, base + space.products, base + space.dw_parts, s);
  if (!large) return launch_linear_tiles_bwd(l, g, dx, dx_accumulate, dw, accumulate, bias, base + space.products, base + space.dw_parts, s);
  if (db) {
    ProfScope prof(MOE_K_LINEAR_BIAS, s);
    hipLaunchKernelGGL(bias_grad, dim3(bias_blocks(l.N, l.e_cnt)), dim3(BIAS_THREADS), 0, s, bias);
    HIP_CHECK_LAUNCH();
  }
  return launch_linear_bwd_large(l, g, dx, dx_accumulate, dw, accumulate, setup, base + space.products, s);
}
