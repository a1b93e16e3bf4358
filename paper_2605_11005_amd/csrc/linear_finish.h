// What the linear layer's kernels do with finished sums: 16 bytes of outputs at a time (bf16: eight columns of a row, fp32: four), and the launches that
// add up a contraction's parts.
#pragma once
#include "activation.h"
#include "linear.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

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
template <typename T>
__device__ __forceinline__ void add_from(const void* p, size_t at, float (&y)[VEC<T>]) {
  float v[VEC<T>];
  values(*reinterpret_cast<const u32x4*>((const T*)p + at), v);
#pragma unroll
  for (int j = 0; j < VEC<T>; ++j) y[j] += v[j];
}
template <typename T>
__device__ __forceinline__ void store_to(void* p, size_t at, const float (&y)[VEC<T>]) {
  *reinterpret_cast<u32x4*>((T*)p + at) = words(y);
}

// From sums with their bias: z is stored, and they become act(z)
template <typename T>
__device__ __forceinline__ void activate_forward(const LinearArgs& l, size_t at, float (&y)[VEC<T>]) {
  if (l.z) store_to<T>(l.z, at, y);
  with_activation(l.act, [&](auto a) {
#pragma unroll
    for (int j = 0; j < VEC<T>; ++j) y[j] = act_value<decltype(a)::value, sizeof(T) == 2>(y[j]);
  });
}
// The forward's outputs at element `at`, columns col and on, of expert e from the sums
template <typename T>
__device__ __forceinline__ void finish_forward(const LinearArgs& l, int e, size_t at, int col, float (&y)[VEC<T>]) {
  if (l.bias) add_from<T>(l.bias, (size_t)e * l.N + col, y);
  activate_forward<T>(l, at, y);
  if (l.residual) add_from<T>(l.residual, at, y);
  store_to<T>(l.y, at, y);
}

// Sums of a contraction's parts: [parts] of the whole output, stride elements apart, added in ascending order
struct Parts {
  float* sums;
  size_t stride;
  int n;                   // 1: not cut, no sums
};
// A weight gradient's contraction, an expert's rows, is cut in up to a launch's n parts.  Grouped, in as many as leave each some rows: experts differ, and
// only the device knows how.
template <typename T>
__device__ __forceinline__ int parts_of_expert(bool grouped, int rows, int n) {
  return grouped ? max(1, min(n, rows / (sizeof(T) == 2 ? 512 : 256))) : n;
}
// What a launch of that is planned for: an expert of six times the mean rows.  Backward, us, without such parts / with them: 32 experts of 96 to 120 with 9953
// rows, 7393 of them one's, 81 / 30 in bf16, 96 / 37 in fp32; 4000, 100 and 20 rows of 1024 to 512 55 / 40 and 174 / 96; 8 experts' 37527 rows of 112
// to 296, 20928 of them one's, 83 / 52 and 255 / 124; all alike, where the launch behind finds nothing to add: 16 experts' 300 rows of 256 to 256 20.2 / 23.8
// and 27.0 / 29.2, 8 experts' 1000 of 512 to 1024 35.5 / 37.8.
inline long long longest_rows(const LinearArgs& l) {
  const long long six = 6ll * ((l.rows + l.e_cnt - 1) / l.e_cnt);
  return l.offsets && six < l.rows ? six : l.rows;
}
template <int V>
__device__ __forceinline__ void add_parts(const Parts& p, size_t at, float (&y)[V]) {
  const float* s = p.sums + at;
  f32x4 v[V / 4];
#pragma unroll
  for (int k = 0; k < V / 4; ++k) v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int q = 0; q < p.n; ++q, s += p.stride)
#pragma unroll
    for (int k = 0; k < V / 4; ++k) v[k] += *reinterpret_cast<const f32x4*>(s + 4 * k);
#pragma unroll
  for (int j = 0; j < V; ++j) y[j] = v[j / 4][j % 4];
}

// A block finishes 128 columns of 2 V rows of an expert.
constexpr int JOIN_THREADS = 256, JOIN_COLUMNS = 128;
template <typename T>
__global__ __launch_bounds__(JOIN_THREADS) void join_forward(LinearArgs l, Parts p) {
  constexpr int V = VEC<T>, LANES = JOIN_COLUMNS / V, ROWS = JOIN_THREADS / LANES;
  const int cols = (l.N + JOIN_COLUMNS - 1) / JOIN_COLUMNS;
  int e = 0, row_tile = blockIdx.x / cols, col_tile = blockIdx.x % cols, row = 0, end = l.rows;
  if (l.offsets) {
    if (!RaggedTiles<ROWS>(l.offsets, l.e_cnt, threadIdx.x & 63).tile(cols, blockIdx.x, e, row_tile, col_tile)) return;
    row = l.offsets[e];
    end = l.offsets[e + 1];
  }
  row += row_tile * ROWS + threadIdx.x / LANES;
  const int col = col_tile * JOIN_COLUMNS + V * (threadIdx.x % LANES);
  if (row >= end || col >= l.N) return;
  const size_t at = (size_t)row * l.N + col;
  float y[V];
  add_parts(p, at, y);
  finish_forward<T>(l, e, at, col, y);
}
template <typename T>
int launch_join_forward(const LinearArgs& l, const Parts& p, hipStream_t s) {
  if (p.n <= 1) return MOE_OK;
  constexpr int ROWS = JOIN_THREADS / (JOIN_COLUMNS / VEC<T>);
  const long long m = ((long long)l.rows + ROWS - 1) / ROWS + (l.offsets ? (l.e_cnt < l.rows ? l.e_cnt : l.rows) - 1 : 0);
  const long long blocks = (m * ((l.N + JOIN_COLUMNS - 1) / JOIN_COLUMNS) + 7) / 8 * 8;
  hipLaunchKernelGGL(join_forward<T>, dim3((unsigned)blocks), dim3(JOIN_THREADS), 0, s, l, p);
  HIP_CHECK_LAUNCH();
  return MOE_OK;
}

// dx of all rows of all experts, and dW of all matrices; what was not cut has no part in it
template <typename T>
__global__ __launch_bounds__(JOIN_THREADS) void join_gradients(LinearArgs l, Parts px, T* dx, int dx_accumulate, Parts pw, T* dw,
                                                            int accumulate) {
  constexpr int V = VEC<T>;
  const size_t rows = l.offsets ? (size_t)l.offsets[l.e_cnt] : (size_t)l.rows;
  const size_t n_dx = px.n > 1 ? rows * l.K / V : 0, n_dw = pw.n > 1 ? (size_t)l.e_cnt * l.K * l.N / V : 0;
  for (size_t v = (size_t)blockIdx.x * JOIN_THREADS + threadIdx.x; v < n_dx + n_dw; v += (size_t)gridDim.x * JOIN_THREADS) {
    float y[V];
    if (v < n_dx) {
      add_parts(px, V * v, y);
      if (dx_accumulate) add_from<T>(dx, V * v, y);
      store_to<T>(dx, V * v, y);
    } else {
      const size_t at = V * (v - n_dx);
      Parts p = pw;
      if (l.offsets) {
        const size_t e = at / ((size_t)l.K * l.N);
        p.n = parts_of_expert<T>(true, l.offsets[e + 1] - l.offsets[e], pw.n);
        if (p.n == 1) continue;                    // (finished by its tiles)
      }
      add_parts(p, at, y);
      if (accumulate) add_from<T>(dw, at, y);
      store_to<T>(dw, at, y);
    }
  }
}
template <typename T>
int launch_join_gradients(const LinearArgs& l, const Parts& px, void* dx, int dx_accumulate, const Parts& pw, void* dw, int accumulate, hipStream_t s) {
  if (px.n <= 1 && pw.n <= 1) return MOE_OK;
  const long long n = ((px.n > 1 ? (long long)l.rows * l.K : 0) + (pw.n > 1 ? (long long)l.e_cnt * l.K * l.N : 0)) / VEC<T>;
  const long long blocks = (n + JOIN_THREADS - 1) / JOIN_THREADS, most = 8ll * device_cu_count();
  ProfScope prof(MOE_K_WGRAD_REDUCE, s);
  hipLaunchKernelGGL(join_gradients<T>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(JOIN_THREADS), 0, s, l, px, (T*)dx, dx_accumulate, pw, (T*)dw,
                     accumulate);
  HIP_CHECK_LAUNCH();
  return MOE_OK;
}

// What adding up the parts of n outputs takes, in us: a launch, and their bytes through the caches
inline float join_time(int parts, double n) { return parts > 1 ? 3.f + (float)(parts * n * (8.0 / 9e6)) : 0.f; }

// Where contractions are cut there are at most this many workgroups; a part's sums of a whole output of rows x columns, for any number of rows up to
// this one, take at most linear_parts_bytes
constexpr int MOST_PARTS = 16, CUT_WORKGROUPS = 512;

}  // namespace
