// The norms between two blocks in one pass: a block's output y is normalised and weighted, gated and added to the residual stream, and the
// sum is normalised for the next block.
//     u = (post_norm ? y r_post : y) w_post       h' = alpha h + beta g[t] u       n = h' r_pre w_pre       r = (mean x^2 + eps)^-1/2
// and its gradient
//     gh = dh' + r_pre (w_pre dn) - h' r_pre^3 mean(w_pre dn h')       dh = alpha gh       du = beta g gh
//     dy = r_post (w_post du) - y r_post^3 mean(w_post du y)           dg = beta sum gh u
//     dw_pre = sum_t dn h' r_pre                                       dw_post = sum_t du y r_post
// HBM bound.  A row stays in the registers of its threads from the load to the store, 16 bytes of y (bf16: eight elements, fp32:
// four) per thread and step, so that every tensor crosses memory once; sums are fp32.
#include "common.h"
#include "kernels.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

template <typename T> constexpr int VEC = 16 / sizeof(T);

// N elements as floats
template <int N>
__device__ __forceinline__ void unpack(const bf16_t* p, size_t i, float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N / 8; ++j) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p + i + 8 * j);
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[8 * j + 2 * k] = bf16lo(w[k]); v[8 * j + 2 * k + 1] = bf16hi(w[k]); }
  }
}
template <int N>
__device__ __forceinline__ void unpack(const float* p, size_t i, float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p + i + 4 * j);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[4 * j + k] = __uint_as_float(w[k]);
  }
}
template <int N>
__device__ __forceinline__ void pack(bf16_t* p, size_t i, const float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N / 8; ++j) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = pack_bf16x2(v[8 * j + 2 * k], v[8 * j + 2 * k + 1]);
    *reinterpret_cast<u32x4*>(p + i + 8 * j) = w;
  }
}
template <int N>
__device__ __forceinline__ void pack(float* p, size_t i, const float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __float_as_uint(v[4 * j + k]);
    *reinterpret_cast<u32x4*>(p + i + 4 * j) = w;
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
// most threads of a row (d up to 16384): fp32 with four steps of four elements takes 1024
template <typename T, int STEPS> constexpr int MOST_THREADS = sizeof(T) == 4 && STEPS == 4 ? 1024 : 512;

template <typename T, typename R>
struct FwdArgs {
  const T* y; const float* gate; const T* w_post; const R* h; const T* w_pre;
  R* h_out; T* n; float* r_post; float* r_pre;
  int T_, d, post_norm;
  float alpha, beta, eps;
};

// A block per row, or (blockDim.y rows) a wavefront per row.
template <typename T, typename R, int STEPS>
__global__ __launch_bounds__((MOST_THREADS<T, STEPS>)) void block_norm_fwd(FwdArgs<T, R> p) {
  constexpr int N = VEC<T>;
  __shared__ float red[2][MOST_WAVES];
  const int row = blockIdx.x * blockDim.y + threadIdx.y;
  RowSum row_total{red, (int)blockDim.x >> 6};
  if (row >= p.T_) return;
  const size_t at = (size_t)row * p.d;
  float v[STEPS][N], h[STEPS][N];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
#pragma unroll
    for (int j = 0; j < N; ++j) v[i][j] = h[i][j] = 0.f;
    if (c < p.d) {
      unpack(p.h, at + c, h[i]);
      if (p.y) unpack(p.y, at + c, v[i]);
    }
  }
  const float inv_d = 1.f / (float)p.d;
  if (p.y) {
    float scale = p.beta * (p.gate ? p.gate[row] : 1.f);
    if (p.post_norm) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) sum += v[i][j] * v[i][j];
      const float r = 1.f / sqrtf(row_total(sum) * inv_d + p.eps);
      if (p.r_post && threadIdx.x == 0) p.r_post[row] = r;
      scale *= r;
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * N;
      float w[N];
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = 1.f;
      if (p.w_post && c < p.d) unpack(p.w_post, c, w);
#pragma unroll
      for (int j = 0; j < N; ++j) h[i][j] = p.alpha * h[i][j] + scale * v[i][j] * w[j];
      if (p.h_out && c < p.d) pack(p.h_out, at + c, h[i]);
    }
  }
  if (!p.w_pre) return;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < STEPS; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) sum += h[i][j] * h[i][j];
  const float r = 1.f / sqrtf(row_total(sum) * inv_d + p.eps);
  if (p.r_pre && threadIdx.x == 0) p.r_pre[row] = r;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
    if (c >= p.d) continue;
    float w[N];
    unpack(p.w_pre, c, w);
#pragma unroll
    for (int j = 0; j < N; ++j) h[i][j] *= r * w[j];
    pack(p.n, at + c, h[i]);
  }
}

template <typename T, typename R>
struct BwdArgs {
  const T* y; const float* gate; const T* w_post; const R* h; const T* w_pre;
  const float* r_post; const float* r_pre;
  const R* dh_out; const T* dn;
  R* dh; T* dy; float* dgate;
  float* sums;                             // [blocks][2][d]: dw_post, dw_pre
  int T_, d, post_norm;
  float alpha, beta;
};

// Blocks walk the rows b, b + grid, .. and keep the column sums of theirs in registers.
template <typename T, typename R, int STEPS>
__global__ __launch_bounds__((MOST_THREADS<T, STEPS>)) void block_norm_bwd(BwdArgs<T, R> p) {
  constexpr int N = VEC<T>;
  __shared__ float red[2][MOST_WAVES];
  RowSum row_total{red, (int)blockDim.x >> 6};
  const float inv_d = 1.f / (float)p.d;
  float w_pre[STEPS][N], w_post[STEPS][N], d_pre[STEPS][N], d_post[STEPS][N];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
#pragma unroll
    for (int j = 0; j < N; ++j) { w_pre[i][j] = d_pre[i][j] = d_post[i][j] = 0.f; w_post[i][j] = 1.f; }
    if (p.w_pre && c < p.d) unpack(p.w_pre, c, w_pre[i]);
    if (p.w_post && c < p.d) unpack(p.w_post, c, w_post[i]);
  }
  for (int row = blockIdx.x; row < p.T_; row += gridDim.x) {
    const size_t at = (size_t)row * p.d;
    float y[STEPS][N], g[STEPS][N];
    {
      float h[STEPS][N], dn[STEPS][N];
      float sum = 0.f;
      const float r = p.w_pre ? p.r_pre[row] : 0.f;
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * N;
#pragma unroll
        for (int j = 0; j < N; ++j) y[i][j] = g[i][j] = h[i][j] = dn[i][j] = 0.f;
        if (c < p.d) {
          if (p.w_pre) { unpack(p.h, at + c, h[i]); unpack(p.dn, at + c, dn[i]); }
          if (p.dh_out) unpack(p.dh_out, at + c, g[i]);
          if (p.y) unpack(p.y, at + c, y[i]);
        }
      }
      if (p.w_pre) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
          for (int j = 0; j < N; ++j) {
            d_pre[i][j] += dn[i][j] * h[i][j] * r;
            dn[i][j] *= w_pre[i][j];
            sum += dn[i][j] * h[i][j];
          }
        const float m = row_total(sum) * inv_d * r * r * r;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
          for (int j = 0; j < N; ++j) g[i][j] += r * dn[i][j] - m * h[i][j];
      }
    }
    if (p.dh) {
      const float alpha = p.y ? p.alpha : 1.f;
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * N;
        float o[N];
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = alpha * g[i][j];
        if (c < p.d) pack(p.dh, at + c, o);
      }
    }
    if (!p.y) continue;
    const float gate = p.gate ? p.gate[row] : 1.f, r = p.post_norm ? p.r_post[row] : 1.f, scale = p.beta * gate * r;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        d_post[i][j] += scale * g[i][j] * y[i][j];
        g[i][j] *= w_post[i][j];
        sum += g[i][j] * y[i][j];
      }
    float m = 0.f;
    if (p.post_norm || p.dgate) {
      const float total = row_total(sum);
      if (p.dgate && threadIdx.x == 0) p.dgate[row] = p.beta * r * total;
      if (p.post_norm) m = scale * r * r * total * inv_d;
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * N;
#pragma unroll
      for (int j = 0; j < N; ++j) g[i][j] = scale * g[i][j] - m * y[i][j];
      if (c < p.d) pack(p.dy, at + c, g[i]);
    }
  }
  float* const out = p.sums + (size_t)blockIdx.x * 2 * p.d;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
    if (c >= p.d) continue;
    if (p.y) pack(out, c, d_post[i]);
    if (p.w_pre) pack(out + p.d, c, d_pre[i]);
  }
}

// The blocks' column sums in ascending order: wavefront w of 16 adds the w-th part of them, 64 columns a block.
constexpr int SUM_WAVES = 16;
template <typename T>
__global__ __launch_bounds__(SUM_WAVES * WAVE) void column_sums(const float* __restrict__ sums, int blocks, int d, int accumulate, T* __restrict__ dw_post,
                                                                T* __restrict__ dw_pre) {
  __shared__ float part[SUM_WAVES][WAVE];
  T* const out = blockIdx.y ? dw_pre : dw_post;
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
  if constexpr (sizeof(T) == 2) out[c] = f32_to_bf16(accumulate ? bf16_to_f32(out[c]) + s : s);
  else out[c] = accumulate ? out[c] + s : s;
}

// threads of a row at `steps` vectors each, whole wavefronts
inline int row_threads(int vecs, int steps) { return WAVE * ((vecs + WAVE * steps - 1) / (WAVE * steps)); }

template <typename T, typename R>
int forward(FwdArgs<T, R> p, hipStream_t s) {
  const int vecs = p.d / VEC<T>;
  int steps = 1;
  while (row_threads(vecs, steps) > 512 && steps < 4) steps *= 2;
  const int threads = row_threads(vecs, steps), rows = threads == WAVE ? 4 : 1;
  const dim3 grid((p.T_ + rows - 1) / rows), block(threads, rows);
  if (steps == 1) hipLaunchKernelGGL((block_norm_fwd<T, R, 1>), grid, block, 0, s, p);
  else if (steps == 2) hipLaunchKernelGGL((block_norm_fwd<T, R, 2>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((block_norm_fwd<T, R, 4>), grid, block, 0, s, p);
  HIP_CHECK_LAUNCH();
  return MOE_OK;
}

constexpr int BWD_BLOCKS = 512;
inline int bwd_blocks(int T) { return T < BWD_BLOCKS ? T : BWD_BLOCKS; }

template <typename T, typename R>
int backward(BwdArgs<T, R> p, T* dw_post, T* dw_pre, int accumulate, hipStream_t s) {
  const int vecs = p.d / VEC<T>, blocks = bwd_blocks(p.T_);
  int steps = 1;
  while (row_threads(vecs, steps) > 512 && steps < 4) steps *= 2;
  const dim3 grid(blocks), block(row_threads(vecs, steps));
  if (p.T_ > 0) {
    ProfScope prof(MOE_K_NORM_BWD, s);
    if (steps == 1) hipLaunchKernelGGL((block_norm_bwd<T, R, 1>), grid, block, 0, s, p);
    else if (steps == 2) hipLaunchKernelGGL((block_norm_bwd<T, R, 2>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((block_norm_bwd<T, R, 4>), grid, block, 0, s, p);
    HIP_CHECK_LAUNCH();
  }
  if (dw_post || dw_pre) {
    ProfScope prof(MOE_K_NORM_SUMS, s);
    hipLaunchKernelGGL(column_sums<T>, dim3((p.d + WAVE - 1) / WAVE, 2), dim3(SUM_WAVES * WAVE), 0, s, p.sums, blocks, p.d, accumulate, dw_post, dw_pre);
    HIP_CHECK_LAUNCH();
  }
  return MOE_OK;
}

template <typename F>
int by_types(int dtype, int res_dtype, F f) {
  if (dtype == MOE_F32) return f((float*)nullptr, (float*)nullptr);
  if (res_dtype == MOE_F32) return f((bf16_t*)nullptr, (float*)nullptr);
  return f((bf16_t*)nullptr, (bf16_t*)nullptr);
}

}  // namespace

size_t block_norm_ws_bytes(int T, int d) { return (size_t)bwd_blocks(T) * 2 * d * sizeof(float); }

int launch_block_norm_fwd(const void* y, const float* gate, const void* w_post, int post_norm, const void* h, const void* w_pre, int dtype, int res_dtype,
                          int T, int d, float alpha, float beta, float eps, void* h_out, void* n, float* r_post, float* r_pre, hipStream_t s) {
  if (T == 0) return MOE_OK;
  ProfScope prof(MOE_K_NORM_FWD, s);
  return by_types(dtype, res_dtype, [&](auto* t, auto* r) {
    typedef std::remove_pointer_t<decltype(t)> X;
    typedef std::remove_pointer_t<decltype(r)> R;
    return forward(FwdArgs<X, R>{(const X*)y, gate, (const X*)w_post, (const R*)h, (const X*)w_pre, (R*)h_out, (X*)n, r_post, r_pre, T, d, post_norm,
                                 alpha, beta, eps}, s);
  });
}

int launch_block_norm_bwd(const void* y, const float* gate, const void* w_post, int post_norm, const void* h_out, const void* w_pre,
                          const float* r_post, const float* r_pre, const void* dh_out, const void* dn, int dtype, int res_dtype, int T, int d,
                          float alpha, float beta, void* dh, void* dy, float* dgate, void* dw_post, void* dw_pre, int accumulate, void* ws,
                          hipStream_t s) {
  return by_types(dtype, res_dtype, [&](auto* t, auto* r) {
    typedef std::remove_pointer_t<decltype(t)> X;
    typedef std::remove_pointer_t<decltype(r)> R;
    return backward(BwdArgs<X, R>{(const X*)y, gate, (const X*)w_post, (const R*)h_out, (const X*)w_pre, r_post, r_pre, (const R*)dh_out, (const X*)dn,
                                  (R*)dh, (X*)dy, dgate, (float*)ws, T, d, post_norm, alpha, beta}, (X*)dw_post, (X*)dw_pre, accumulate, s);
  });
}
