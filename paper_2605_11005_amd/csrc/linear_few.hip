// The linear layer's forward with few rows per matrix, in bf16: y = act(x W[e] + b[e]) + residual, bound by reading the weights once.
//
// A workgroup multiplies up to 64 rows of one expert by a strip of 128 columns, over the contraction or a part of it; its four wavefronts
// share that, 32 k at a time in turn, and their sums meet in LDS in ascending order.  Weights go from memory to the matrix instruction
// through registers alone: a lane loads 16 bytes of each of eight rows, eight columns by eight k (Piece, few_rows.h), and column j of that block
// is its operand of the j-th of eight 16x16x32 instructions, in which row i of the instruction stands for column 8 i + j of the strip.  The sums
// of a lane's eight instructions are then eight consecutive columns of one row of x.
// A CU takes in about 33 GB/s of weights however many of its wavefronts ask for them, so what counts is how many CUs ask: few strips
// are cut along the contraction (plan()), each part stores fp32 sums, and a second launch adds them in order and finishes them.
#include "few_rows.h"
#include "linear_finish.h"

namespace {

constexpr int STRIP = 128, DEPTH = 2, PITCH = STRIP + 4, W = 4, TM = 64;

struct FewArgs {
  LinearArgs l;
  Parts parts;
  int part_steps;          // steps of 32 k of a part
};

// The expert (e), rows [row0, row0 + rows) and strip of a launch's tile `b`; false: the list is shorter.  An expert's tiles are listed by strip, row
// tiles fastest: those of a strip read the same weights.
struct Place { int e, row0, rows, n0; };
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

template <int TG, bool STREAM>
__device__ __forceinline__ void few_tile(const FewArgs& p, const Place& at, int part, float (*sums)[16][PITCH]) {
  const LinearArgs& l = p.l;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int K = l.K, N = l.N, rows = at.rows, first = part * p.part_steps, steps = min((K + KP - 1) / KP, first + p.part_steps);
  const bf16_t* const w = (const bf16_t*)l.w + (size_t)at.e * K * N + at.n0;
  const bf16_t* const x = (const bf16_t*)l.x + (size_t)at.row0 * K;
  const int wcol = 2 * min(8 * i, N - at.n0 - 8);          // columns and rows past the end repeat the last ones
  int xrow[TG];
#pragma unroll
  for (int t = 0; t < TG; ++t) xrow[t] = 2 * min(16 * t + i, rows - 1) * K;
  Piece piece[DEPTH];
  u32x4 xs[DEPTH][TG];
  auto load = [&](auto slot, int step) {
    constexpr int S = decltype(slot)::value;
    const bool in = step < steps;
    const int from = in ? step : 0, k = min(8 * g, K - 8 - KP * from);     // chunks past the contraction's end repeat its last one
    piece[S].template load<0, 8, STREAM>(w + (size_t)from * KP * N, in, 2 * N, 2 * k * N + wcol);
    const __amdgpu_buffer_rsrc_t d = descriptor(x + from * KP, in);
#pragma unroll
    for (int t = 0; t < TG; ++t) xs[S][t] = __builtin_amdgcn_raw_buffer_load_b128(d, xrow[t] + 2 * k, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  f32x4 acc[8][TG];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int t = 0; t < TG; ++t) acc[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](auto slot, int step) {
    constexpr int S = decltype(slot)::value;
    if (KP * (step + 1) > K && KP * step + 8 * g >= K) {                 // (of either operand: the other may be no number)
#pragma unroll
      for (int r = 0; r < 8; ++r) piece[S].w[r] = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int t = 0; t < TG; ++t) xs[S][t] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
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
      for (int r = 0; r < 4; ++r) {                        // element r of acc[j][t]: column 8 (4 g + r) + j, row 16 t + i
        float* const to = &sums[wave][i][8 * (4 * g + r)];
        *reinterpret_cast<f32x4*>(to) = f32x4{acc[0][t][r], acc[1][t][r], acc[2][t][r], acc[3][t][r]};
        *reinterpret_cast<f32x4*>(to + 4) = f32x4{acc[4][t][r], acc[5][t][r], acc[6][t][r], acc[7][t][r]};
      }
    }
    __syncthreads();
    const int row = threadIdx.x / (STRIP / 8), c = 8 * (threadIdx.x % (STRIP / 8)), col = at.n0 + c;
    if (16 * t + row < rows && col < N) {
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

template <bool STREAM>
__global__ __launch_bounds__(W * WAVE, 2) void linear_few(FewArgs p) {
  __shared__ __align__(16) float sums[W][16][PITCH];
  static_assert(W * WAVE == 16 * STRIP / 8, "a thread finishes eight columns of a row");
  Place at;
  if (!place_of(p.l, blockIdx.x, threadIdx.x & 63, at)) return;
  if (at.rows <= 16) few_tile<1, STREAM>(p, at, blockIdx.y, sums);
  else if (at.rows <= 32) few_tile<2, STREAM>(p, at, blockIdx.y, sums);
  else few_tile<4, STREAM>(p, at, blockIdx.y, sums);
}

#ifndef FEW_PARTS
#define FEW_PARTS 0
#endif
// tiles of 64 rows by a strip, at most
inline long long tiles_of(int rows, int N, int e_cnt) {
  return (((long long)rows + TM - 1) / TM + (e_cnt < rows ? e_cnt : rows) - 1) * ((N + STRIP - 1) / STRIP);
}
inline int parts_of(int rows, int K, int N, int e_cnt) {
  if (FEW_PARTS) return FEW_PARTS;
  // us: weights at what memory delivers or at what the CU with the most strips takes in, and the launch that adds the parts up
  const long long tiles = tiles_of(rows, N, e_cnt);
  const int steps = (K + KP - 1) / KP;
  const double memory = (double)(e_cnt < rows ? e_cnt : rows) * K * N * (2 / 6.5e6);
  double best = 0;
  int parts = 1;
  for (int p = 1; p <= MOST_PARTS && p <= steps / (2 * W) && (p == 1 || p * tiles <= CUT_WORKGROUPS); ++p) {
    const double cu = (double)((p * tiles + 255) / 256) * ((steps + p - 1) / p) * (KP * 2 * STRIP / 40e3);
    const double t = (cu > memory ? cu : memory) + join_time(p, (double)rows * N);
    if (p == 1 || t < best) { best = t; parts = p; }
  }
  return parts;
}

}  // namespace

// parts * rows * N floats for any number of rows up to this one: parts is at most MOST_PARTS, and CUT_WORKGROUPS strips of 64 rows
size_t linear_few_ws_bytes(int rows, int N) {
  const size_t all = (size_t)MOST_PARTS * rows * N * 4, most = (size_t)CUT_WORKGROUPS * TM * STRIP * 4;
  return all < most ? all : most;
}

int launch_linear_few(const LinearArgs& l, void* ws, hipStream_t s) {
  const int steps = (l.K + KP - 1) / KP, parts = parts_of(l.rows, l.K, l.N, l.e_cnt), per = (steps + parts - 1) / parts;
  const FewArgs p = {l, {(float*)ws, (size_t)l.rows * l.N, (steps + per - 1) / per}, per};
  const dim3 grid((unsigned)((tiles_of(l.rows, l.N, l.e_cnt) + 7) / 8 * 8), p.parts.n);
  ProfScope prof(MOE_K_LINEAR, s);
  // (stream_rule.h: weights that the Infinity Cache does not keep)
  if (2ll * l.K * l.N * l.e_cnt > (256ll << 20)) hipLaunchKernelGGL(linear_few<true>, grid, dim3(W * WAVE), 0, s, p);
  else hipLaunchKernelGGL(linear_few<false>, grid, dim3(W * WAVE), 0, s, p);
  HIP_CHECK_LAUNCH();
  return launch_join_forward<bf16_t>(l, p.parts, s);
}
