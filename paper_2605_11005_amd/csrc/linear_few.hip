// The linear layer's forward with few rows per matrix, in bf16: y = act(x W[e] + b[e]) + residual, bound by reading the weights once.
//
// A workgroup multiplies up to 64 rows of one expert by a strip of 128 columns, or 64, over the contraction or a part of it; its four wavefronts
// share that, 32 k at a time in turn, and their sums meet in LDS in ascending order.  Weights go from memory to the matrix instruction
// through registers alone: a lane loads C = 8 (or 4) columns of each of eight rows, and column j of that block is its operand of the j-th of C
// 16x16x32 instructions, in which row i of the instruction stands for column C i + j of the strip.  The sums of a lane's C instructions
// are then C consecutive columns of one row of x.
// What a CU takes in of weights does not go by how many of its wavefronts ask for them: 33 GB/s with 4, 8 and 16 wavefronts for each of 112 strips (4 rows of
// 4096 to 14336, 31 to 33 us), 44 GB/s where 32 CUs have a strip each (14336 to 4096, 83 us).  So what counts is how many CUs ask: narrower strips, or
// strips cut along the contraction, whose parts store fp32 sums that a second launch adds in order and finishes (plan_of).
#include "linear_finish.h"
#include "linear_piece.h"

namespace {

constexpr int DEPTH = 2, W = 4, TM = 64, KP = 32;
constexpr long long PART_SUMS = 4 << 20;       // of all parts together, at most

struct FewArgs {
  LinearArgs l;
  Parts parts;
  int part_steps;          // steps of 32 k of a part
};

// The expert (e), rows [row0, row0 + rows) and strip of a launch's tile `b`; false: the list is shorter.  An expert's tiles are listed by strip, row
// tiles fastest: those of a strip read the same weights.
struct Place { int e, row0, rows, n0; };
template <int STRIP>
__device__ __forceinline__ bool place_of(const LinearArgs& l, int b, int lane, Place& at) {
  const int strips = (l.N + STRIP - 1) / STRIP;
  int e = 0, first = 0, end = l.rows, line, strip, row_tile;
  if (l.offsets) {
    int col;
    if (!RaggedTiles<TM>(l.offsets, l.e_cnt, lane).tile(strips, b, e, line, col)) return false;
    first = l.offsets[e];
    end = l.offsets[e + 1];
    line = line * strips + col;
  } else {
    const int total = (l.rows + TM - 1) / TM * strips, share = (total + 7) / 8;
    line = (b % 8) * share + b / 8;
    if (b / 8 >= share || line >= total) return false;
  }
  const int m = (end - first + TM - 1) / TM;
  strip = line / m;
  row_tile = line - strip * m;
  at.e = __builtin_amdgcn_readfirstlane(e);
  at.row0 = __builtin_amdgcn_readfirstlane(first + row_tile * TM);
  at.rows = __builtin_amdgcn_readfirstlane(min(TM, end - first - row_tile * TM));
  at.n0 = __builtin_amdgcn_readfirstlane(strip * STRIP);
  return true;
}

template <int C, int TG, bool STREAM>
__device__ __forceinline__ void few_tile(const FewArgs& p, const Place& at, int part, float (*sums)[16][16 * C + 4]) {
  constexpr int STRIP = 16 * C;
  const LinearArgs& l = p.l;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int K = l.K, N = l.N, rows = at.rows, first = part * p.part_steps, steps = min((K + KP - 1) / KP, first + p.part_steps);
  const bf16_t* const w = (const bf16_t*)l.w + (size_t)at.e * K * N + at.n0;
  const bf16_t* const x = (const bf16_t*)l.x + (size_t)at.row0 * K;
  const int wcol = 2 * min(C * i, N - at.n0 - C);          // columns and rows past the end repeat the last ones
  int xrow[TG];
#pragma unroll
  for (int t = 0; t < TG; ++t) xrow[t] = 2 * min(16 * t + i, rows - 1) * K;
  ColumnPiece<C> piece[DEPTH];
  u32x4 xs[DEPTH][TG];
  auto load = [&](auto slot, int step) {
    constexpr int S = decltype(slot)::value;
    const bool in = step < steps;
    const int from = in ? step : 0, k = min(8 * g, K - 8 - KP * from);     // chunks past the contraction's end repeat its last one
    piece[S].template load<STREAM>(w + (size_t)from * KP * N, in, 2 * N, 2 * k * N + wcol);
    const __amdgpu_buffer_rsrc_t d = descriptor(x + from * KP, in);
#pragma unroll
    for (int t = 0; t < TG; ++t) xs[S][t] = __builtin_amdgcn_raw_buffer_load_b128(d, xrow[t] + 2 * k, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  f32x4 acc[C][TG];
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int t = 0; t < TG; ++t) acc[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](auto slot, int step) {
    constexpr int S = decltype(slot)::value;
    if (KP * (step + 1) > K && KP * step + 8 * g >= K) {                 // (of either operand: the other may be no number)
#pragma unroll
      for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int q = 0; q < C / 2; ++q) piece[S].w[r][q] = 0;
#pragma unroll
      for (int t = 0; t < TG; ++t) xs[S][t] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const bf16x8 f = piece[S].operand(j);
#pragma unroll
      for (int t = 0; t < TG; ++t) acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, __builtin_bit_cast(bf16x8, xs[S][t]), acc[j][t], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  static_for<DEPTH>([&](auto s) { load(s, first + wave + W * decltype(s)::value); });
  for (int step = first + wave; step < steps; step += W * DEPTH)
    static_for<DEPTH>([&](auto s) {
      constexpr int S = decltype(s)::value;
      multiply(s, step + W * S);
      load(s, step + W * (S + DEPTH));
    });
#pragma unroll
  for (int t = 0; t < TG; ++t) {
    if (16 * t >= rows) break;
    if (t) __syncthreads();
    if (16 * t + i < rows) {
#pragma unroll
      for (int r = 0; r < 4; ++r)                          // element r of acc[j][t]: column C (4 g + r) + j, row 16 t + i
#pragma unroll
        for (int j = 0; j < C; j += 4)
          *reinterpret_cast<f32x4*>(&sums[wave][i][C * (4 * g + r) + j]) = f32x4{acc[j][t][r], acc[j + 1][t][r], acc[j + 2][t][r], acc[j + 3][t][r]};
    }
    __syncthreads();
    const int row = threadIdx.x / (STRIP / 8), c = 8 * (threadIdx.x % (STRIP / 8)), col = at.n0 + c;
    if (row < 16 && 16 * t + row < rows && col < N) {
      f32x4 lo = f32x4{0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll
      for (int q = 0; q < W; ++q) {
        lo += *reinterpret_cast<const f32x4*>(&sums[q][row][c]);
        hi += *reinterpret_cast<const f32x4*>(&sums[q][row][c + 4]);
      }
      const int to = at.row0 + 16 * t + row;
      const size_t out = (size_t)to * N + col;
      if (p.parts.n > 1) {
        float* const s = p.parts.sums + part * p.parts.stride + out;
        *reinterpret_cast<f32x4*>(s) = lo;
        *reinterpret_cast<f32x4*>(s + 4) = hi;
      } else {
        float y[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        finish_forward<bf16_t>(l, at.e, out, col, y);
      }
    }
  }
}

template <int C, bool STREAM>
__global__ __launch_bounds__(W * WAVE, 2) void linear_few(FewArgs p) {
  __shared__ __align__(16) float sums[W][16][16 * C + 4];
  static_assert(W * WAVE >= 16 * 16 * C / 8, "a thread finishes eight columns of a row");
  Place at;
  if (!place_of<16 * C>(p.l, blockIdx.x, threadIdx.x & 63, at)) return;
  if (at.rows <= 16) few_tile<C, 1, STREAM>(p, at, blockIdx.y, sums);
  else if (at.rows <= 32) few_tile<C, 2, STREAM>(p, at, blockIdx.y, sums);
  else few_tile<C, 4, STREAM>(p, at, blockIdx.y, sums);
}

inline long long strips_of(int N, int strip) { return (N + strip - 1) / strip; }
// tiles of 64 rows by a strip, at most
inline long long most_tiles(int rows, int N, int e_cnt, int strip) {
  return (((long long)rows + TM - 1) / TM + (e_cnt < rows ? e_cnt : rows) - 1) * strips_of(N, strip);
}
// Time in us of strips of `bytes` each: what memory delivers, or what the CU with the most strips takes in, less of it while all CUs ask; and the first
// loads of each
inline float strips_time(long long strips, float bytes, float chip, float cu) {
  const float rounds = (float)((strips + 255) / 256), memory = (float)strips * bytes / chip, own = rounds * bytes / (strips > 256 ? 0.71f * cu : cu);
  return 0.5f * rounds + (memory > own ? memory : own);
}
// Columns of a lane and parts of the contraction, by their time and that of the launch that adds the parts up.  How many experts have rows is not
// known here: the mean over counts from half of what may to all.  Rows of 64 columns come a little slower, from memory and into a CU.  (45 GB/s into a CU
// is what few strips get; for 112 whole ones the model says 24 us where 32 are measured, and cuts them all the same.)
// One row, us, strips of 128 whole / of 64 whole / of 128 in two parts / in eight: 4096 to 14336 31.9 / 26.8 / 25.8 / 26.0; 14336 to 4096 82.8 / 61.1 / 48.4
// / 26.6; 4096 to 1536 17.3 / 13.4 / 12.6 / 8.4; 768 to 4096 5.6 / 5.2 / 7.6 / 7.7.  128 rows of 32 experts of 7168 to 2048, strips of 128 whole / in two /
// in four: 14 of them with rows 70.7 / 75.9 / 77.8, 16 75.9 / 77.4 / 81.3, 17 119.9 / 98.2 / 91.6, 20 119.6 / 102.1 / 99.7, 24 126 / 114 / 117, 32
// 147 / 146 / 150.
struct Plan { int c, parts; };
inline Plan plan_of(int rows, int K, int N, int e_cnt) {
  const int steps = (K + KP - 1) / KP, all = e_cnt < rows ? e_cnt : rows, half = (all + 1) / 2, samples = all - half < 7 ? all - half + 1 : 8;
  const long long row_tiles = ((long long)rows + TM - 1) / TM;
  float best = 0;
  Plan plan = {0, 0};
  for (int c = 8; c >= 4; c -= 4) {
    const int strip = 16 * c;
    const float chip = c == 8 ? 6.5e6f : 5.5e6f, cu = c == 8 ? 45e3f : 33e3f;
    for (int p = 1; p <= MOST_PARTS && p <= steps / (2 * W) && (p == 1 || (long long)p * rows * N <= PART_SUMS); ++p) {
      const float bytes = (float)((steps + p - 1) / p) * (float)(KP * 2 * strip);
      float t = 0.f;
      for (int i = 0; i < samples; ++i) {
        const int active = samples > 1 ? half + (int)((long long)i * (all - half) / (samples - 1)) : all;
        t += strips_time(p * (active > row_tiles ? active : row_tiles) * strips_of(N, strip), bytes, chip, cu);
      }
      t = t / (float)samples + join_time(p, (double)rows * N);
      if (plan.c == 0 || t < 0.97f * best) { best = t; plan = {c, p}; }
    }
    if (plan.c == 0) { plan = {8, 1}; break; }             // (a contraction too short to be cut)
  }
  return plan;
}

}  // namespace

// parts * rows * N floats for any number of rows up to this one
size_t linear_few_ws_bytes(int rows, int N) {
  const size_t all = (size_t)MOST_PARTS * rows * N;
  return 4 * (all < PART_SUMS ? all : PART_SUMS);
}

int launch_linear_few(const LinearArgs& l, void* ws, hipStream_t s) {
  const Plan plan = plan_of(l.rows, l.K, l.N, l.e_cnt);
  const int steps = (l.K + KP - 1) / KP, per = (steps + plan.parts - 1) / plan.parts;
  const FewArgs p = {l, {(float*)ws, (size_t)l.rows * l.N, (steps + per - 1) / per}, per};
  const dim3 grid((unsigned)((most_tiles(l.rows, l.N, l.e_cnt, 16 * plan.c) + 7) / 8 * 8), p.parts.n);
  ProfScope prof(MOE_K_LINEAR, s);
  const bool stream = 2ll * l.K * l.N * l.e_cnt > (256ll << 20);       // (stream_rule.h: weights that the Infinity Cache does not keep)
  const auto kernel = plan.c == 8 ? (stream ? linear_few<8, true> : linear_few<8, false>) : (stream ? linear_few<4, true> : linear_few<4, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(W * WAVE), 0, s, p);
  HIP_CHECK_LAUNCH();
  return launch_join_forward<bf16_t>(l, p.parts, s);
}
