// Layer norm between two blocks in one pass: a block's output is added to the residual stream, and the sum is normalised for the next one.
//     h' = h + y        n = (h' - mean) rstd w + b        rstd = (mean (h' - mean)^2 + eps)^-1/2
// and its gradient, with t = w dn and xh = (h' - mean) rstd,
//     dh = dh' + rstd (t - mean t - xh mean(t xh))        dw = sum_t dn xh        db = sum_t dn
// HBM bound.  A row stays in the registers of its threads, 16 bytes of y or n per thread and step, so that every tensor crosses memory once.
// The squares are of what is left of a value after its mean: a row whose mean is large beside its deviation keeps its digits.  Each wavefront
// takes its own mean first, and the wavefronts' sums and squares join behind one barrier: with counts c_w, means m_w and squares q_w,
//     sum (x - mean)^2 = sum_w q_w + c_w (m_w - mean)^2.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "norm_rows.h"

namespace {

// Threads of a row's elements (d up to 16384): fp32 with four steps of four elements takes 1024.
template <typename T, int STEPS> constexpr int MOST_THREADS = sizeof(T) == 4 && STEPS == 4 ? 1024 : 512;

template <typename T, typename R>
struct FwdArgs {
  const T* y; const R* h; const T* w; const T* b;
  R* h_out; T* n; float* mean; float* rstd;
  int T_, d;
  float eps;
  int row0;                                // of this launch
};

// A block per row, or (blockDim.y rows) a wavefront per row.  STREAM: y is loaded and n stored as not used again soon.
template <typename T, typename R, int STEPS, bool STREAM>
__global__ __launch_bounds__((MOST_THREADS<T, STEPS>)) void layer_norm_fwd(FwdArgs<T, R> p) {
  constexpr int N = VEC<T>;
  __shared__ float2 red[MOST_WAVES];
  const int row = p.row0 + blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= p.T_) return;                 // (a block of several rows has no barrier)
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
  const size_t at = (size_t)row * p.d;
  float h[STEPS][N];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
    float y[N];
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = h[i][j] = 0.f;
    if (c < p.d) {
      unpack(p.h, at + c, h[i]);
      if (p.y) unpack<N, STREAM>(p.y, at + c, y);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) h[i][j] += y[j];
    if (p.y && p.h_out && c < p.d) pack(p.h_out, at + c, h[i]);
  }
  // of wavefront w: its elements, in all steps
  const auto count = [&](int w) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) n += max(0, min(WAVE * N, p.d - (int)(i * blockDim.x + w * WAVE) * N));
    return (float)n;
  };
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < STEPS; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) sum += h[i][j];
  sum = wave_total(sum);
  float mean = sum / fmaxf(count(wave), 1.f), squares = 0.f;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const bool in = (int)(i * blockDim.x + threadIdx.x) * N < p.d;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float v = h[i][j] - mean;
      squares += in ? v * v : 0.f;
    }
  }
  squares = wave_total(squares);
  const float inv_d = 1.f / (float)p.d;
  if (waves > 1) {
    if ((threadIdx.x & 63) == 0) red[wave] = make_float2(sum, squares);
    __syncthreads();
    sum = squares = 0.f;
    for (int w = 0; w < waves; ++w) sum += red[w].x;
    mean = sum * inv_d;
    for (int w = 0; w < waves; ++w) {
      const float n = count(w), off = red[w].x / fmaxf(n, 1.f) - mean;
      squares += red[w].y + n * off * off;
    }
  }
  const float rstd = 1.f / sqrtf(squares * inv_d + p.eps);
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
    if (c >= p.d) continue;
    float w[N], b[N];
#pragma unroll
    for (int j = 0; j < N; ++j) { w[j] = 1.f; b[j] = 0.f; }
    if (p.w) unpack(p.w, c, w);
    if (p.b) unpack(p.b, c, b);
#pragma unroll
    for (int j = 0; j < N; ++j) h[i][j] = (h[i][j] - mean) * rstd * w[j] + b[j];
    pack<N, STREAM>(p.n, at + c, h[i]);
  }
}

template <typename T, typename R>
struct BwdArgs {
  const R* h; const T* w; const float* mean; const float* rstd;
  const R* dh_out; const T* dn;
  R* dh; T* dy;
  float* sums;                             // [blocks][2][d]: dw, db
  int T_, d;
};

// What the backward reads of a row
template <typename T, typename R, int STEPS, bool STREAM>
struct BwdRow {
  static constexpr int N = VEC<T>;
  Raw<T, N> dn[STEPS];
  Raw<R, N> h[STEPS], dh[STEPS];
  float mean, rstd;
  __device__ __forceinline__ void load(const BwdArgs<T, R>& p, int row) {
    const size_t at = (size_t)row * p.d;
    mean = rstd = 0.f;
    if (row < p.T_) { mean = p.mean[row]; rstd = p.rstd[row]; }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * N;
      dn[i].clear(); h[i].clear(); dh[i].clear();
      if (row < p.T_ && c < p.d) {
        h[i].template load<STREAM>(p.h, at + c);
        dn[i].template load<STREAM>(p.dn, at + c);
        if (p.dh_out) dh[i].template load<STREAM>(p.dh_out, at + c);
      }
    }
  }
};

// Blocks (or, for rows of one wavefront, wavefronts) walk the rows and keep the column sums of theirs in registers; the next row's loads are on
// their way while a row's sums meet.  For WIDE rows the registers hold neither these nor the weights, and the column sums are in LDS.
// STREAM: inputs beyond what the Infinity Cache holds are loaded as used once (streams()).
constexpr int BWD_ROWS = 8, BWD_THREADS = 512, WIDE_THREADS = 1024;
template <typename T, typename R, int STEPS, bool WIDE, bool STREAM>
__global__ __launch_bounds__(WIDE ? WIDE_THREADS : BWD_THREADS) void layer_norm_bwd(BwdArgs<T, R> p) {
  constexpr int N = VEC<T>;
  __shared__ float2 red[2][MOST_WAVES];
  const int waves = blockDim.x >> 6;
  int turn = 0;
  const float inv_d = 1.f / (float)p.d;
  Raw<T, N> w_raw[STEPS];
  float dw[STEPS][N], db[STEPS][N];
  extern __shared__ f32x4 column_lds[];               // WIDE: [dw, db][step][four columns][thread]
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
    w_raw[i].clear();
#pragma unroll
    for (int j = 0; j < N; ++j) dw[i][j] = db[i][j] = 0.f;
    if constexpr (WIDE)
#pragma unroll
      for (int q = 0; q < N / 4; ++q) column(0, i, q) = column(1, i, q) = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!WIDE && p.w && c < p.d) w_raw[i].load(p.w, c);
  }
  BwdRow<T, R, STEPS, STREAM> next;
  int row = blockIdx.x * blockDim.y + threadIdx.y;
  if (!WIDE) next.load(p, row);
  for (; row < p.T_; row += gridDim.x * blockDim.y) {
    const size_t at = (size_t)row * p.d;
    float xh[STEPS][N], t[STEPS][N], g[STEPS][N];
    if (WIDE) next.load(p, row);
    const float mean = next.mean, rstd = next.rstd;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) { next.dn[i].values(t[i]); next.h[i].values(xh[i]); next.dh[i].values(g[i]); }
    if (!WIDE) next.load(p, row + gridDim.x * blockDim.y);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * N;
      float w[N], v[N];
      if (WIDE && p.w && c < p.d) w_raw[i].load(p.w, c);
      w_raw[i].values(w);
      add(1, i, db[i], t[i]);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        xh[i][j] = (xh[i][j] - mean) * rstd;
        v[j] = t[i][j] * xh[i][j];
        if (p.w) t[i][j] *= w[j];
        s1 += t[i][j];
        s2 += t[i][j] * xh[i][j];
      }
      add(0, i, dw[i], v);
    }
    s1 = wave_total(s1);
    s2 = wave_total(s2);
    if (waves > 1) {                       // (two places in turn: one is written again only behind the barrier of the row in between)
      float2* const place = red[turn];
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) place[threadIdx.x >> 6] = make_float2(s1, s2);
      __syncthreads();
      s1 = s2 = 0.f;
      for (int k = 0; k < waves; ++k) { s1 += place[k].x; s2 += place[k].y; }
    }
    s1 *= inv_d;
    s2 *= inv_d;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * N;
#pragma unroll
      for (int j = 0; j < N; ++j) g[i][j] += rstd * (t[i][j] - s1 - xh[i][j] * s2);
      if (c < p.d) {
        if (p.dh) pack(p.dh, at + c, g[i]);
        if (p.dy) pack(p.dy, at + c, g[i]);
      }
    }
  }
  if constexpr (!WIDE && STEPS * N <= 16)
    if (blockDim.y > 1) {                  // a block's wavefronts' sums, in their order
      __shared__ float part[BWD_ROWS][N][WAVE];
#pragma unroll
      for (int k = 0; k < 2 * STEPS; ++k) {
        float(&v)[N] = k % 2 ? db[k / 2] : dw[k / 2];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j) part[threadIdx.y][j][threadIdx.x] = v[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j) {
          v[j] = 0.f;
          for (int q = 0; q < (int)blockDim.y; ++q) v[j] += part[q][j][threadIdx.x];
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
      for (int j = 0; j < N; ++j) { dw[i][j] = column(0, i, j / 4)[j % 4]; db[i][j] = column(1, i, j / 4)[j % 4]; }
    pack(out, c, dw[i]);
    pack(out + p.d, c, db[i]);
  }
}

// The backward of few rows in one launch: blocks of rows as in the forward, and blocks that sum 64 columns over all rows, for which dw and db need the saved
// mean and 1/deviation alone.  What the latter read again comes from the caches.  DEEP, from several hundred rows on: the blocks that sum begin first and have
// eight rows a thread on their way, and may sum a part of the rows each, which a second launch adds up.
constexpr int SUM_COLUMNS = 64, SUM_AHEAD = 8, PART_ROWS = 256;
template <typename T, typename R>
struct OneLaunch {
  BwdArgs<T, R> p;
  T* dw; T* db;
  int accumulate, row_blocks;
  int parts;                               // DEEP: of the rows; more than one leave their sums in p.sums
};
template <bool DEEP, typename T, typename R>
__device__ __forceinline__ void sum_columns(const OneLaunch<T, R>& a, int c0, int row_part) {
  constexpr int N = VEC<T>, LANES = SUM_COLUMNS / N, AT_ONCE = WAVE / LANES;      // lanes and rows of a wavefront's load
  __shared__ float part[2][MOST_WAVES][SUM_COLUMNS];
  const BwdArgs<T, R>& p = a.p;
  const int tid = threadIdx.y * blockDim.x + threadIdx.x, waves = blockDim.x * blockDim.y >> 6, wave = tid >> 6, lane = tid & 63;
  const int c = c0 + lane % LANES * N;
  float dw[N], db[N];
#pragma unroll
  for (int j = 0; j < N; ++j) dw[j] = db[j] = 0.f;
  if constexpr (DEEP) {
    const int share = (p.T_ + a.parts - 1) / a.parts, end = min(p.T_, (row_part + 1) * share), stride = waves * AT_ONCE;
    if (c < p.d)
      for (int first = row_part * share + wave * AT_ONCE + lane / LANES; first < end; first += SUM_AHEAD * stride) {
        Raw<R, N> h[SUM_AHEAD];
        Raw<T, N> dn[SUM_AHEAD];
        float mean[SUM_AHEAD], rstd[SUM_AHEAD];
#pragma unroll
        for (int u = 0; u < SUM_AHEAD; ++u) {              // (rows past the end: the first one again, and left out)
          const int row = first + u * stride < end ? first + u * stride : first;
          h[u].load(p.h, (size_t)row * p.d + c);
          dn[u].load(p.dn, (size_t)row * p.d + c);
          mean[u] = p.mean[row];
          rstd[u] = p.rstd[row];
        }
#pragma unroll
        for (int u = 0; u < SUM_AHEAD; ++u) {
          const bool in = first + u * stride < end;
          float x[N], g[N];
          h[u].values(x);
          dn[u].values(g);
#pragma unroll
          for (int j = 0; j < N; ++j) {
            dw[j] += in ? g[j] * ((x[j] - mean[u]) * rstd[u]) : 0.f;
            db[j] += in ? g[j] : 0.f;
          }
        }
      }
  } else if (c < p.d)
#pragma unroll 4
    for (int row = wave * AT_ONCE + lane / LANES; row < p.T_; row += waves * AT_ONCE) {
      float h[N], dn[N];
      unpack(p.h, (size_t)row * p.d + c, h);
      unpack(p.dn, (size_t)row * p.d + c, dn);
      const float mean = p.mean[row], rstd = p.rstd[row];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        dw[j] += dn[j] * ((h[j] - mean) * rstd);
        db[j] += dn[j];
      }
    }
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int m = LANES; m < WAVE; m *= 2) {
      dw[j] += __shfl_xor(dw[j], m);
      db[j] += __shfl_xor(db[j], m);
    }
  if (lane < LANES)
#pragma unroll
    for (int j = 0; j < N; ++j) { part[0][wave][lane * N + j] = dw[j]; part[1][wave][lane * N + j] = db[j]; }
  __syncthreads();
  for (int i = tid; i < 2 * SUM_COLUMNS; i += 64 * waves) {        // (a block may be a single wavefront)
    const int which = i / SUM_COLUMNS, col = i % SUM_COLUMNS;
    T* const out = which ? a.db : a.dw;
    if (!out || c0 + col >= p.d) continue;
    float s = 0.f;
    for (int w = 0; w < waves; ++w) s += part[which][w][col];
    if (DEEP && a.parts > 1) {
      p.sums[((size_t)row_part * 2 + which) * p.d + c0 + col] = s;
      continue;
    }
    T& to = out[c0 + col];
    if constexpr (sizeof(T) == 2) to = (bf16_t)pack_bf16x2(a.accumulate ? bf16_to_f32(to) + s : s, 0.f);      // (the hardware's conversion keeps every NaN)
    else to = a.accumulate ? to + s : s;
  }
}
template <typename T, typename R, int STEPS, bool DEEP>
__global__ __launch_bounds__((MOST_THREADS<T, STEPS>)) void layer_norm_bwd_few(OneLaunch<T, R> a) {
  constexpr int N = VEC<T>;
  __shared__ float2 red[MOST_WAVES];       // of the block's wavefronts, a row's one after the other
  const BwdArgs<T, R>& p = a.p;
  int block = blockIdx.x;
  if constexpr (DEEP) {
    const int sums = (int)gridDim.x - a.row_blocks;
    if (block < sums) return sum_columns<true>(a, block / a.parts * SUM_COLUMNS, block % a.parts);
    block -= sums;
  } else if (block >= a.row_blocks) return sum_columns<false>(a, (block - a.row_blocks) * SUM_COLUMNS, 0);
  const int row = block * blockDim.y + threadIdx.y;
  const bool in = row < p.T_;
  const size_t at = (size_t)row * p.d;
  const float mean = in ? p.mean[row] : 0.f, rstd = in ? p.rstd[row] : 0.f, inv_d = 1.f / (float)p.d;
  float xh[STEPS][N], t[STEPS][N], g[STEPS][N], s1 = 0.f, s2 = 0.f;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
    float w[N];
#pragma unroll
    for (int j = 0; j < N; ++j) { xh[i][j] = mean; t[i][j] = g[i][j] = 0.f; w[j] = 1.f; }
    if (in && c < p.d) {
      unpack(p.h, at + c, xh[i]);
      unpack(p.dn, at + c, t[i]);
      if (p.dh_out) unpack(p.dh_out, at + c, g[i]);
      if (p.w) unpack(p.w, c, w);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      xh[i][j] = (xh[i][j] - mean) * rstd;
      t[i][j] *= w[j];
      s1 += t[i][j];
      s2 += t[i][j] * xh[i][j];
    }
  }
  s1 = wave_total(s1);
  s2 = wave_total(s2);
  const int waves = blockDim.x >> 6;
  if (waves > 1) {
    float2* const mine = red + threadIdx.y * waves;
    if ((threadIdx.x & 63) == 0) mine[threadIdx.x >> 6] = make_float2(s1, s2);
    __syncthreads();
    s1 = s2 = 0.f;
    for (int k = 0; k < waves; ++k) { s1 += mine[k].x; s2 += mine[k].y; }
  }
  s1 *= inv_d;
  s2 *= inv_d;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * N;
    if (!in || c >= p.d) continue;
#pragma unroll
    for (int j = 0; j < N; ++j) g[i][j] += rstd * (t[i][j] - s1 - xh[i][j] * s2);
    if (p.dh) pack(p.dh, at + c, g[i]);
    if (p.dy) pack(p.dy, at + c, g[i]);
  }
}

// Threads and steps of a row, rows of a block
struct Shape {
  int steps, threads, rows;
  Shape(int d, int vec) {
    const int vecs = d / vec;
    steps = 1;
    while (row_threads(vecs, steps) > 512 && steps < 4) steps *= 2;
    if (vecs > WAVE && vecs <= 3 * WAVE / 2) steps = 2;
    threads = row_threads(vecs, steps);
    rows = threads == WAVE ? 4 : 1;
  }
  dim3 block() const { return dim3(threads, rows); }
};
template <typename T, typename R>
int forward(FwdArgs<T, R> p, hipStream_t s) {
  const Shape shape(p.d, VEC<T>);
  const int steps = shape.steps, threads = shape.threads, rows = shape.rows;
  const dim3 block = shape.block();
  // STREAM of tensors beyond the Infinity Cache, us, as usual / so: 32768 rows of 7168 bf16 with fp32 residuals 510 / 503, 16384 of 4096 140 / 138, of bf16
  // 96 / 93, 65536 of 1024 94 / 87; within it 16384 of 1024 23.3 / 24.9.  Hints on the residual stream cost up to a tenth.
  const bool stream = (double)p.T_ * p.d * 2 * (sizeof(T) + sizeof(R)) > (double)(256ll << 20);
  const auto of = [&](auto st) {
    constexpr bool STREAM = decltype(st)::value != 0;
    return steps == 1 ? layer_norm_fwd<T, R, 1, STREAM> : steps == 2 ? layer_norm_fwd<T, R, 2, STREAM> : layer_norm_fwd<T, R, 4, STREAM>;
  };
  const auto kernel = stream ? of(Int<1>{}) : of(Int<0>{});
  return in_launches(((long long)p.T_ + rows - 1) / rows, threads * rows, [&](long long first, unsigned blocks) {
    p.row0 = (int)first * rows;
    hipLaunchKernelGGL(kernel, dim3(blocks), block, 0, s, p);
  });
}

// The backward's launch: rows of up to 16 elements a lane in one wavefront, several of them in a block; longer rows in a block each.
struct BwdPlan { int steps, threads, rows, most, blocks; bool wide; };
// Nontemporal loads of more than the Infinity Cache holds, us, as usual / so: 16384 rows of 4096 bf16 107 / 93, of 7168 174 / 154, 65536 of 1024
// 103 / 90; of less: 2047 of 2880 16.5 / 19.4, 16384 of 1024 30.0 / 30.9.  Fewer rows at a time then do: 16384 of 4096 bf16 in one block of 512
// threads per CU 89, with fp32 residuals 206 -> 197 (but fp32, eight elements a thread less, 16384 of 2048 88 -> 106); 32768 of 2048 in two blocks of
// 256 per CU for four 98 -> 92.
// Within the cache too one block per CU does where its loads alone keep the CU busy, and where rows are so few that the blocks' sums count, us, two / one:
// 8192 of 4096 bf16 54.0 / 48.4, 2047 19.6 / 17.9 (of 3584 45.2 / 46.4 and 18.5 / 17.5), with fp32 residuals 12000 of 2048 85 / 73, 4096 of 2880 37.3 / 35.3
// (of 1536 22.0 / 24.3); 1100 of 1536 12.1 / 11.4, of 2880 15.4 / 13.6 (4096 of 2880 23.0 / 25.1).
inline bool streams(int T, int d, int element, int residual, bool through) {
  return (double)T * d * (element + residual * (through ? 2 : 1)) > (double)(256ll << 20);
}
inline BwdPlan bwd_plan(int T, int d, int vec, bool fp32_residual, bool stream) {
  constexpr int CUS = 256;
  const int vecs = d / vec, per = 16 / vec;          // steps of 16 elements
  BwdPlan b;
  b.wide = row_threads(vecs, per) > BWD_THREADS;
  if (row_threads(vecs, 1) == WAVE) b.steps = 1;
  else if (b.wide || row_threads(vecs, per) == WAVE) b.steps = per;
  else b.steps = row_threads(vecs, 1) <= BWD_THREADS ? 1 : row_threads(vecs, 2) <= BWD_THREADS ? 2 : per;
  b.threads = row_threads(vecs, b.steps);
  const bool fills = vec == 8 && (b.threads > 448 || (b.threads > 256 && stream) || (b.threads >= 256 && fp32_residual));
  const int per_cu = b.steps * vec == 16 || fills || (b.threads > 2 * WAVE && T <= 6 * CUS) ? 1 : !stream && b.threads > WAVE && b.threads <= 256 && T >= 8192 ? 4 : 2;
  b.most = T < per_cu * CUS ? T : per_cu * CUS;
  b.rows = b.threads > WAVE ? 1 : T >= per_cu * CUS * BWD_ROWS ? BWD_ROWS : T == 0 ? 1 : (T - 1) / (per_cu * CUS) + 1;
  const int units = T == 0 ? 0 : (T - 1) / b.rows + 1;
  b.blocks = units < b.most ? units : b.most;
  return b;
}

// Two launches / one / one, DEEP, us: 256 rows of 2880 bf16 9.5 / 5.2 / 5.8, of 16384 21.8 / 12.5 / 12.2, 512 of 7168 17.2 / 11.7 / 10.4, 700 of 520 - / 5.2 / 6.4,
// 1000 of 2880 - / 12.5 / 10.0, of 4096 16.3 / 12.7 / 10.7, with fp32 residuals 19.5 / 20.1 / 16.2, of 7168 18.9 / - / 15.9 (27.4 / - / 28.8).  Two / DEEP, in
// parts: 1100 of 520 15.1 / 7.6, 4096 13.2 / 10.3, 2047 of 1032 13.3 / 11.5 (4096 of 1032 16.9 / 18.5, 2047 of 2880 16.6 / 20.7, 10000
// of 128 with fp32 residuals 12.4 / 14.5).
enum class FewRows { NO, SHALLOW, DEEP };
inline FewRows few_rows(int T, int d, int element, int residual) {
  const long long n = (long long)T * d;
  if (T > 1024) return T <= 4096 && n * residual <= (8ll << 20) ? FewRows::DEEP : FewRows::NO;
  if (T > 512 && n * (element + residual) > (30ll << 20)) return FewRows::NO;
  return T >= 700 && n >= 1600000 ? FewRows::DEEP : FewRows::SHALLOW;
}

template <typename T, typename R>
int add_columns(const BwdArgs<T, R>& p, int blocks, T* dw, T* db, int accumulate, hipStream_t s) {
  if (!dw && !db) return MOE_OK;
  ProfScope prof(MOE_K_LAYER_NORM_SUMS, s);
  hipLaunchKernelGGL(column_sums<T>, dim3((p.d + WAVE - 1) / WAVE, 2), dim3(SUM_WAVES * WAVE), 0, s, p.sums, blocks, p.d, accumulate, dw, db);
  HIP_CHECK_LAUNCH();
  return MOE_OK;
}
template <typename T, typename R>
int backward(BwdArgs<T, R> p, T* dw, T* db, int accumulate, hipStream_t s) {
  // (in place, the rows would write over what the column sums still read)
  const auto over = [&](const void* out) { return out && (out == p.dn || out == p.h); };
  const bool in_place = (dw || db) && (over(p.dh) || over(p.dy));
  const FewRows few = p.T_ == 0 || in_place ? FewRows::NO : few_rows(p.T_, p.d, sizeof(T), sizeof(R));
  if (few != FewRows::NO) {
    Shape shape(p.d, VEC<T>);
    if (shape.threads < 512) shape.rows = 512 / shape.threads;      // (the blocks that sum columns want wavefronts)
    const int parts = p.T_ <= 1024 ? 1 : (p.T_ + PART_ROWS - 1) / PART_ROWS;       // at most 16
    const OneLaunch<T, R> a = {p, dw, db, accumulate, p.dh || p.dy ? (p.T_ + shape.rows - 1) / shape.rows : 0, parts};
    const unsigned blocks = a.row_blocks + (dw || db ? parts * ((p.d + SUM_COLUMNS - 1) / SUM_COLUMNS) : 0);
    if (blocks == 0) return MOE_OK;
    {
      ProfScope prof(MOE_K_LAYER_NORM_BWD, s);
      const auto of = [&](auto deep) {
        constexpr bool DEEP = decltype(deep)::value != 0;
        return shape.steps == 1 ? layer_norm_bwd_few<T, R, 1, DEEP> : shape.steps == 2 ? layer_norm_bwd_few<T, R, 2, DEEP> : layer_norm_bwd_few<T, R, 4, DEEP>;
      };
      hipLaunchKernelGGL(few == FewRows::DEEP ? of(Int<1>{}) : of(Int<0>{}), dim3(blocks), shape.block(), 0, s, a);
      HIP_CHECK_LAUNCH();
    }
    return parts > 1 ? add_columns(p, parts, dw, db, accumulate, s) : MOE_OK;
  }
  const bool stream = streams(p.T_, p.d, sizeof(T), sizeof(R), p.dh_out);
  const BwdPlan plan = bwd_plan(p.T_, p.d, VEC<T>, sizeof(R) == 4, stream);
  const int steps = plan.steps, blocks = plan.blocks;
  const dim3 grid(blocks), block(plan.threads, plan.rows);
  constexpr int PER = 16 / VEC<T>;
  if (p.T_ > 0) {
    ProfScope prof(MOE_K_LAYER_NORM_BWD, s);
    if (plan.wide) {
      const size_t lds = 2 * sizeof(float) * 16 * plan.threads;
      static bool attr_set[64] = {};
      int dev = 0;
      if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return MOE_EHIP;
      if (!attr_set[dev]) {
        for (const void* kernel : {reinterpret_cast<const void*>(&layer_norm_bwd<T, R, PER, true, false>), reinterpret_cast<const void*>(&layer_norm_bwd<T, R, PER, true, true>)})
          if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * sizeof(float) * 16 * WIDE_THREADS) != hipSuccess) return MOE_EHIP;
        attr_set[dev] = true;
      }
      const auto kernel = stream ? layer_norm_bwd<T, R, PER, true, true> : layer_norm_bwd<T, R, PER, true, false>;
      hipLaunchKernelGGL(kernel, grid, block, lds, s, p);
    } else {
      const auto of = [&](auto st) {
        constexpr bool STREAM = decltype(st)::value != 0;
        return steps == 1 ? layer_norm_bwd<T, R, 1, false, STREAM> : steps == 2 ? layer_norm_bwd<T, R, 2, false, STREAM> : layer_norm_bwd<T, R, PER, false, STREAM>;
      };
      hipLaunchKernelGGL(stream ? of(Int<1>{}) : of(Int<0>{}), grid, block, 0, s, p);
    }
    HIP_CHECK_LAUNCH();
  }
  return add_columns(p, blocks, dw, db, accumulate, s);
}

}  // namespace

// For T rows and fewer, of bf16 or fp32
size_t layer_norm_ws_bytes(int T, int d) {
  int most = 0;
  for (int vec : {8, 4})
    for (bool fp32 : {false, true})
      for (bool stream : {false, true}) most = std::max(most, bwd_plan(T, d, vec, fp32, stream).most);
  return (size_t)most * 2 * d * sizeof(float);
}

int launch_layer_norm_fwd(const void* y, const void* h, const void* w, const void* b, int dtype, int res_dtype, int T, int d, float eps, void* h_out,
                          void* n, float* mean, float* rstd, hipStream_t s) {
  if (T == 0) return MOE_OK;
  ProfScope prof(MOE_K_LAYER_NORM_FWD, s);
  return by_types(dtype, res_dtype, [&](auto* t, auto* r) {
    typedef std::remove_pointer_t<decltype(t)> X;
    typedef std::remove_pointer_t<decltype(r)> R;
    return forward(FwdArgs<X, R>{(const X*)y, (const R*)h, (const X*)w, (const X*)b, (R*)h_out, (X*)n, mean, rstd, T, d, eps}, s);
  });
}

int launch_layer_norm_bwd(const void* h_out, const void* w, const float* mean, const float* rstd, const void* dh_out, const void* dn, int dtype,
                          int res_dtype, int T, int d, void* dh, void* dy, void* dw, void* db, int accumulate, void* ws, hipStream_t s) {
  return by_types(dtype, res_dtype, [&](auto* t, auto* r) {
    typedef std::remove_pointer_t<decltype(t)> X;
    typedef std::remove_pointer_t<decltype(r)> R;
    return backward(BwdArgs<X, R>{(const R*)h_out, (const X*)w, mean, rstd, (const R*)dh_out, (const X*)dn, (R*)dh, (X*)dy, (float*)ws, T, d},
                    (X*)dw, (X*)db, accumulate, s);
  });
}
