// The norms between two blocks in one pass: a block's output y is normalised and weighted, gated and added to the residual stream, and the
// sum is normalised for the next block.
//     u = (post_norm ? y r_post : y) w_post       h' = alpha h + beta g[t] u       n = h' r_pre w_pre       r = (mean x^2 + eps)^-1/2
// and its gradient
//     gh = dh' + r_pre (w_pre dn) - h' r_pre^3 mean(w_pre dn h')       dh = alpha gh       du = beta g gh
//     dy = r_post (w_post du) - y r_post^3 mean(w_post du y)           dg = beta sum gh u
//     dw_pre = sum_t dn h' r_pre                                       dw_post = sum_t du y r_post
// HBM bound.  A row stays in the registers of its threads from the load to the store, 16 bytes of y (bf16: eight elements, fp32:
// four) per thread and step, so that every tensor crosses memory once; sums are fp32.  Measured, of 6.5 TB/s that a copy reaches: forward of
// 32768 rows of 7168 (y, n bf16, h fp32) 495 us, 5.7 TB/s; backward of 16384 rows of 4096 (h fp32) 229 us, 5.3 TB/s, of 32768 rows of 7168 bf16 523 us,
// 5.4 TB/s; the forward of four rows takes 1 us over an empty launch.  Hints that data are not used again cost the forward a tenth.
#include "common.h"
#include "kernels.h"
#include "norm_rows.h"

namespace {

// most threads of a row (d up to 16384): fp32 with four steps of four elements takes 1024
template <typename T, int STEPS> constexpr int MOST_THREADS = sizeof(T) == 4 && STEPS == 4 ? 1024 : 512;

template <typename T, typename R>
struct FwdArgs {
  const T* y; const float* gate; const T* w_post; const R* h; const T* w_pre;
  R* h_out; T* n; float* r_post; float* r_pre;
  int T_, d, post_norm;
  float alpha, beta, eps;
  int row0;                                // of this launch
};

// A block per row, or (blockDim.y rows) a wavefront per row.
template <typename T, typename R, int STEPS>
__global__ __launch_bounds__((MOST_THREADS<T, STEPS>)) void block_norm_fwd(FwdArgs<T, R> p) {
  constexpr int N = VEC<T>;
  __shared__ float red[2][MOST_WAVES];
  const int row = p.row0 + blockIdx.x * blockDim.y + threadIdx.y;
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

// What the backward reads of a row
template <typename T, typename R, int STEPS>
struct BwdRow {
  static constexpr int N = VEC<T>;
  Raw<T, N> y[STEPS], dn[STEPS];
  Raw<R, N> h[STEPS], dh[STEPS];
  __device__ __forceinline__ void load(const BwdArgs<T, R>& p, int row) {
    const size_t at = (size_t)row * p.d;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * N;
      dn[i].clear(); h[i].clear(); dh[i].clear();
      if (row < p.T_ && c < p.d) {
        if (p.w_pre) { h[i].load(p.h, at + c); dn[i].load(p.dn, at + c); }
        if (p.dh_out) dh[i].load(p.dh_out, at + c);
      }
    }
  }
  __device__ __forceinline__ void load_y(const BwdArgs<T, R>& p, int row) {
    const size_t at = (size_t)row * p.d;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * N;
      y[i].clear();
      if (row < p.T_ && c < p.d && p.y) y[i].load(p.y, at + c);
    }
  }
};

// Blocks (or, for rows of one wavefront, wavefronts) walk the rows and keep the column sums of theirs in registers.  The next row's loads
// are on their way while a row's sums meet; for WIDE rows the registers hold neither these nor the weights, and the column sums are in LDS:
// 4096 rows of 16384 bf16 take 168 to 177 us (4.6 TB/s), fp32, which spills 20 registers, 342 to 352 (4.6 TB/s); with the sums in registers, of which
// 30 to 100 spilled, 240 and 514.
constexpr int BWD_ROWS = 8, BWD_THREADS = 512, WIDE_THREADS = 1024;
template <typename T, typename R, int STEPS, bool WIDE>
__global__ __launch_bounds__(WIDE ? WIDE_THREADS : BWD_THREADS) void block_norm_bwd(BwdArgs<T, R> p) {
  constexpr int N = VEC<T>;
  __shared__ float red[2][MOST_WAVES];
  RowSum row_total{red, (int)blockDim.x >> 6};
  const float inv_d = 1.f / (float)p.d;
  Raw<T, N> w_pre[STEPS], w_post[STEPS];
  float d_pre[STEPS][N], d_post[STEPS][N];
  extern __shared__ f32x4 column_lds[];               // WIDE: [dw_post, dw_pre][step][four columns][thread]
  const auto column = [&](int which, int i, int q) -> f32x4& { return column_lds[((which * STEPS + i) * (N / 4) + q) * blockDim.x + threadIdx.x]; };
  const auto add = [&](int which, int i, float(&sums)[N], const float(&v)[N]) {
    if constexpr (WIDE) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q) column(which, i, q) += f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) sums[j] += v[j];
    }
  };
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
    w_pre[i].clear(); w_post[i].clear();
#pragma unroll
    for (int j = 0; j < N; ++j) d_pre[i][j] = d_post[i][j] = 0.f;
    if constexpr (WIDE)
#pragma unroll
      for (int q = 0; q < N / 4; ++q) column(0, i, q) = column(1, i, q) = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!WIDE && p.w_pre && c < p.d) w_pre[i].load(p.w_pre, c);
    if (!WIDE && p.w_post && c < p.d) w_post[i].load(p.w_post, c);
  }
  BwdRow<T, R, STEPS> next;
  int row = blockIdx.x * blockDim.y + threadIdx.y;
  if (!WIDE) { next.load(p, row); next.load_y(p, row); }
  for (; row < p.T_; row += gridDim.x * blockDim.y) {
    const size_t at = (size_t)row * p.d;
    float y[STEPS][N], g[STEPS][N];
    {
      float h[STEPS][N], dn[STEPS][N];
      if (WIDE) next.load(p, row);
#pragma unroll
      for (int i = 0; i < STEPS; ++i) { if (!WIDE) next.y[i].values(y[i]); next.dn[i].values(dn[i]); next.h[i].values(h[i]); next.dh[i].values(g[i]); }
      const int after = row + gridDim.x * blockDim.y;
      if (!WIDE) { next.load(p, after); next.load_y(p, after); }
      if (p.w_pre) {
        const float r = p.r_pre[row];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const int c = (i * blockDim.x + threadIdx.x) * N;
          float w[N], v[N];
          if (WIDE && c < p.d) w_pre[i].load(p.w_pre, c);
          w_pre[i].values(w);
#pragma unroll
          for (int j = 0; j < N; ++j) {
            v[j] = dn[i][j] * h[i][j] * r;
            dn[i][j] *= w[j];
            sum += dn[i][j] * h[i][j];
          }
          add(1, i, d_pre[i], v);
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
    if (WIDE) {
      next.load_y(p, row);
#pragma unroll
      for (int i = 0; i < STEPS; ++i) next.y[i].values(y[i]);
    }
    const float gate = p.gate ? p.gate[row] : 1.f, r = p.post_norm ? p.r_post[row] : 1.f, scale = p.beta * gate * r;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * N;
      float w[N], v[N];
      if (WIDE && p.w_post && c < p.d) w_post[i].load(p.w_post, c);
      w_post[i].values(w);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        v[j] = scale * g[i][j] * y[i][j];
        if (p.w_post) g[i][j] *= w[j];
        sum += g[i][j] * y[i][j];
      }
      add(0, i, d_post[i], v);
    }
    float m = 0.f;
    if (p.post_norm || p.dgate) {
      const float total = row_total(sum);
      if (p.dgate && threadIdx.x == 0) p.dgate[row] = p.beta * r * total;
      if (p.post_norm) m = total * inv_d * r * r * scale;          // (from the sum on: r^3 of a row of zeros may pass fp32)
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * N;
#pragma unroll
      for (int j = 0; j < N; ++j) g[i][j] = scale * g[i][j] - m * y[i][j];
      if (c < p.d) pack(p.dy, at + c, g[i]);
    }
  }
  if constexpr (!WIDE && STEPS * N <= 16)
    if (blockDim.y > 1) {                  // a block's wavefronts' sums, in their order
      __shared__ float part[BWD_ROWS][N][WAVE];
#pragma unroll
      for (int k = 0; k < 2 * STEPS; ++k) {
        float(&v)[N] = k % 2 ? d_pre[k / 2] : d_post[k / 2];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j) part[threadIdx.y][j][threadIdx.x] = v[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j) {
          v[j] = 0.f;
          for (int w = 0; w < (int)blockDim.y; ++w) v[j] += part[w][j][threadIdx.x];
        }
      }
      if (threadIdx.y) return;
    }
  float* const out = p.sums + (size_t)blockIdx.x * 2 * p.d;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
    if (c >= p.d) continue;
    if constexpr (WIDE)
#pragma unroll
      for (int j = 0; j < N; ++j) { d_post[i][j] = column(0, i, j / 4)[j % 4]; d_pre[i][j] = column(1, i, j / 4)[j % 4]; }
    if (p.y) pack(out, c, d_post[i]);
    if (p.w_pre) pack(out + p.d, c, d_pre[i]);
  }
}

template <typename T, typename R>
int forward(FwdArgs<T, R> p, hipStream_t s) {
  const int vecs = p.d / VEC<T>;
  int steps = 1;
  while (row_threads(vecs, steps) > 512 && steps < 4) steps *= 2;
  // A second wavefront half empty or more costs more than a second step: 65536 rows of 520 bf16 55 us, 74 with two, of 768 72 and 78, of 1024 94
  // and 92.
  if (vecs > WAVE && vecs <= 3 * WAVE / 2) steps = 2;
  const int threads = row_threads(vecs, steps), rows = threads == WAVE ? 4 : 1;
  const dim3 block(threads, rows);
  return in_launches((p.T_ + rows - 1) / rows, threads * rows, [&](long long first, unsigned blocks) {
    p.row0 = (int)first * rows;
    if (steps == 1) hipLaunchKernelGGL((block_norm_fwd<T, R, 1>), dim3(blocks), block, 0, s, p);
    else if (steps == 2) hipLaunchKernelGGL((block_norm_fwd<T, R, 2>), dim3(blocks), block, 0, s, p);
    else hipLaunchKernelGGL((block_norm_fwd<T, R, 4>), dim3(blocks), block, 0, s, p);
  });
}

// The backward's launch.  A thread with one step of bf16 takes 124 registers, with 16 elements up to 252: one block of the latter fits on a
// CU, of the former two.  A row of 1024 elements in one wavefront has no barrier (16384 rows of bf16: 48 us
// against 80 us as blocks of two wavefronts); few rows go to more blocks, not to more wavefronts of a block.  Of blocks of up to 256 threads four fit,
// and from 8192 rows on they are worth twice the column sums: 8192 rows of 1408 bf16 37.5 us, 46.8 with two, 65536 of 2048 320 and 358.
struct BwdPlan { int steps, threads, rows, most, blocks; bool wide; };
inline BwdPlan bwd_plan(int T, int d, int vec) {
  constexpr int CUS = 256;
  const int vecs = d / vec, per = 16 / vec;          // steps of 16 elements
  BwdPlan b;
  b.wide = row_threads(vecs, per) > BWD_THREADS;
  if (row_threads(vecs, 1) == WAVE) b.steps = 1;
  else if (b.wide || row_threads(vecs, per) == WAVE) b.steps = per;
  else b.steps = row_threads(vecs, 1) <= BWD_THREADS ? 1 : row_threads(vecs, 2) <= BWD_THREADS ? 2 : per;
  b.threads = row_threads(vecs, b.steps);
  const int per_cu = b.steps * vec == 16 ? 1 : b.threads > WAVE && b.threads <= 256 && T >= 8192 ? 4 : 2;
  b.most = T < per_cu * CUS ? T : per_cu * CUS;
  b.rows = b.threads > WAVE ? 1 : T >= per_cu * CUS * BWD_ROWS ? BWD_ROWS : T == 0 ? 1 : (T - 1) / (per_cu * CUS) + 1;
  const int units = T == 0 ? 0 : (T - 1) / b.rows + 1;
  b.blocks = units < b.most ? units : b.most;
  return b;
}

template <typename T, typename R>
int backward(BwdArgs<T, R> p, T* dw_post, T* dw_pre, int accumulate, hipStream_t s) {
  const BwdPlan plan = bwd_plan(p.T_, p.d, VEC<T>);
  const int steps = plan.steps, blocks = plan.blocks;
  const dim3 grid(blocks), block(plan.threads, plan.rows);
  constexpr int PER = 16 / VEC<T>;
  if (p.T_ > 0) {
    ProfScope prof(MOE_K_NORM_BWD, s);
    if (plan.wide) {
      const size_t lds = 2 * sizeof(float) * 16 * plan.threads;
      static bool attr_set[64] = {};
      int dev = 0;
      if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return MOE_EHIP;
      if (!attr_set[dev]) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(&block_norm_bwd<T, R, PER, true>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                2 * sizeof(float) * 16 * WIDE_THREADS) != hipSuccess)
          return MOE_EHIP;
        attr_set[dev] = true;
      }
      hipLaunchKernelGGL((block_norm_bwd<T, R, PER, true>), grid, block, lds, s, p);
    }
    else if (steps == 1) hipLaunchKernelGGL((block_norm_bwd<T, R, 1, false>), grid, block, 0, s, p);
    else if (steps == 2) hipLaunchKernelGGL((block_norm_bwd<T, R, 2, false>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((block_norm_bwd<T, R, PER, false>), grid, block, 0, s, p);
    HIP_CHECK_LAUNCH();
  }
  if (dw_post || dw_pre) {
    ProfScope prof(MOE_K_NORM_SUMS, s);
    hipLaunchKernelGGL(column_sums<T>, dim3((p.d + WAVE - 1) / WAVE, 2), dim3(SUM_WAVES * WAVE), 0, s, p.sums, blocks, p.d, accumulate, dw_post, dw_pre);
    HIP_CHECK_LAUNCH();
  }
  return MOE_OK;
}

}  // namespace

// For T rows and fewer, of bf16 or fp32
size_t block_norm_ws_bytes(int T, int d) {
  const int a = bwd_plan(T, d, 8).most, b = bwd_plan(T, d, 4).most;
  return (size_t)(a > b ? a : b) * 2 * d * sizeof(float);
}

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
