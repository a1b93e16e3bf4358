// The linear layer's products in bf16 where the large tiles of expert_bf16.hip would leave most of the chip idle: 128x128 tiles, as many workgroups as
// it takes, contractions in parts.
//     FWD  y  = act(x W + b) + residual    ragged rows, W read transposed
//     DX   dx (+)= dz W^T                  ragged rows, both operands contiguous along the contraction
//     DW   dW (+)= x^T dz                  contraction over an expert's rows, both operands read transposed
// Four wavefronts of 64x64 each, k-tiles 64 deep in two stages of 32 KB, two workgroups per CU: while one waits for its barrier or its operands
// or finishes its outputs, the other multiplies.  A k-tile's fragments are read as a whole, so that its stage is free for the k-tile after the
// next half-way through its multiplication.  Where the tiles alone would not fill the chip the contraction is cut; a part's sums are stored
// in fp32 and added in order by a launch behind (join_forward, join_gradients: linear_finish.h).
// Every output is one chain of sums over ascending k per part.
#include <algorithm>

#include "bias_grad.h"
#include "linear_finish.h"
#include "linear_piece.h"
#include "tile128.h"

namespace {

enum { FWD, DX, DW };
constexpr int NT = 256, TILE_PITCH = 68;
constexpr int STAGE = 2 * QOPER_BYTES, SLAB = 64 * TILE_PITCH * 4;
// tiles of up to 64 rows
constexpr int SHORT = 64, SHORT_A = SHORT * QK * 2, SHORT_STAGE = SHORT_A + QOPER_BYTES, SHORT_DEPTH = 3, SHORT_PITCH = 36;
constexpr int most(int a, int b) { return a > b ? a : b; }
constexpr int TILE_LDS = most(most(4 * SLAB, 2 * STAGE), SHORT_DEPTH * SHORT_STAGE);
static_assert(TILE_LDS <= 80 * 1024, "two workgroups per CU");

// one product: rows [rows of an expert] x N columns (DW: M x N per expert), contraction K (DW: the expert's rows)
struct Product {
  const bf16_t *A, *B;
  long lda, ldb, b_es;
  bf16_t* C;
  int M, N, K;
  Parts parts;
  int accumulate;
  long long tiles;         // at most, of one part (dense: exactly)
};
struct TileArgs {
  LinearArgs l;
  Product p;
};

struct Tile { int e, mt, nt, first, end; };      // rows [first, end) of expert e

// tile b of a part's list: an expert's tiles in bands of 8 row tiles, column tile next, row tile inside the band fastest, so that what an XCD
// multiplies at a time shares panels
template <int OP>
__device__ __forceinline__ bool tile_of(const LinearArgs& l, const Product& p, int b, int part, int lane, Tile& t) {
  const int n_tiles = (p.N + QT - 1) / QT;
  int e = 0, at, m;
  t.first = 0;
  t.end = l.rows;
  if (OP == DW) {
    m = (p.M + QT - 1) / QT;
    // an XCD takes an eighth of the list; where experts differ in rows, every eighth chunk of 32 tiles, of the next part the XCD beside it
    const int total = l.e_cnt * m * n_tiles, share = (total + 7) / 8;
    at = l.offsets ? (b / 256 * 8 + (b + part) % 8) * 32 + b / 8 % 32 : b / 8 < share ? b % 8 * share + b / 8 : total;
    if (at >= total) return false;
    e = at / (m * n_tiles);
    at -= e * m * n_tiles;
    if (l.offsets) { t.first = l.offsets[e]; t.end = l.offsets[e + 1]; }
  } else if (l.offsets) {
    int row_tile, col_tile;
    if (!RaggedTiles<QT>(l.offsets, l.e_cnt, lane).tile(n_tiles, b, e, row_tile, col_tile)) return false;
    t.first = l.offsets[e];
    t.end = l.offsets[e + 1];
    m = (t.end - t.first + QT - 1) / QT;
    at = row_tile * n_tiles + col_tile;
  } else {
    m = (l.rows + QT - 1) / QT;
    const int total = m * n_tiles, share = (total + 7) / 8;
    at = (b % 8) * share + b / 8;
    if (b / 8 >= share || at >= total) return false;
  }
  const int band = at / (8 * n_tiles), in_band = at - band * 8 * n_tiles, high = min(8, m - 8 * band);
  t.nt = __builtin_amdgcn_readfirstlane(in_band / high);
  t.mt = __builtin_amdgcn_readfirstlane(8 * band + in_band % high);
  t.e = __builtin_amdgcn_readfirstlane(e);
  t.first = __builtin_amdgcn_readfirstlane(t.first);
  t.end = __builtin_amdgcn_readfirstlane(t.end);
  return true;
}

// eight finished columns of a row
template <int OP>
__device__ __forceinline__ void finish(const LinearArgs& l, const Product& p, int e, size_t at, int col, float (&y)[8]) {
  if (OP == FWD) return finish_forward<bf16_t>(l, e, at, col, y);
  if (p.accumulate) add_from<bf16_t>(p.C, at, y);
  store_to<bf16_t>(p.C, at, y);
}

// eight columns of a row of a part
template <int OP>
__device__ __forceinline__ void store_out(const LinearArgs& l, const Product& p, int e, int parts, int part, size_t at, int col, const float* from) {
  const f32x4 lo = *reinterpret_cast<const f32x4*>(from), hi = *reinterpret_cast<const f32x4*>(from + 4);
  if (parts > 1) {
    float* const to = p.parts.sums + part * p.parts.stride + at;
    *reinterpret_cast<f32x4*>(to) = lo;
    *reinterpret_cast<f32x4*>(to + 4) = hi;
  } else {
    float y[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    finish<OP>(l, p, e, at, col, y);
  }
}

// Matrices with up to 64 rows, bound by reading the weights: four wavefronts of 64 x 32 and three stages of 24 KB, so that more weights are on their
// way and none are read into registers twice.  Forwards, us, as the other tiles / so: 40 rows of 14336 to 4096 37.0 / 31.5, of 4096 to 14336 36.2 / 32.0,
// eight experts' 20 to 180 rows of 2048 to 1408 24.6 / 22.5, 16 experts' 20 to 306 of 2880 to 2880 75 / 68.  (What an expert of more rows has left over
// past whole tiles reads weights that its other tiles read, from L2: 300 rows each 31.2, so 35.5.)
template <int OP, bool STREAM>
__device__ __forceinline__ void multiply_short(const LinearArgs& l, const Product& p, const Tile& t, int part, char* lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = t.nt * QT, row0 = t.first + t.mt * QT, rows = t.end - row0;
  const int depth = p.K, all = (depth + QK - 1) / QK, per = (all + p.parts.n - 1) / p.parts.n, kt0 = min(all, part * per), kt1 = min(all, kt0 + per);
  const uint32_t base = lds_addr(lds);
  const bf16_t* const A = p.A + (size_t)row0 * p.lda;
  uint32_t a_from[2];                              // load j of a wavefront: rows 8 (2 wave + j) + lane / 8
#pragma unroll
  for (int j = 0; j < 2; ++j) a_from[j] = (uint32_t)(min(8 * (2 * wave + j) + (lane >> 3), rows - 1) * p.lda * 2 + 16 * QuarterKc::chunk(j, lane));
  QuarterKc b_kc;
  QuarterTr b_tr;
  if (OP == FWD) b_tr.setup(p.B + (size_t)t.e * p.b_es, nullptr, false, p.ldb, n0, p.N, wave, lane);
  else b_kc.setup(p.B + (size_t)t.e * p.b_es + (size_t)n0 * p.ldb, p.ldb, p.N - n0, wave, lane);
  auto issue = [&](int kt, int slot) {
    const uint32_t st = base + slot * SHORT_STAGE;
    const long k0 = (long)kt * QK;
    const int last = depth - 1 - (int)k0;          // >= 0
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t back = last < QK - 1 ? past_end((int)k0 + 8 * QuarterKc::chunk(j, lane), depth) : 0;
      if (j < 2) lds_load16(A + k0, a_from[j] - back, st + (2 * wave + j) * 1024);
      if (OP == DX) b_kc.template issue1<STREAM>(j, st + SHORT_A, wave, k0, back);
      else b_tr.template issue1<true, STREAM>(j, st + SHORT_A, wave, lane, k0, last);
    }
  };
  int a_off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = i * 32 + (lane & 31);
    a_off[i] = row * 128 + (((lane >> 5) ^ ((row >> 1) & 7)) << 4);
  }
  const int col = wave * 32 + (lane & 31);
  const int b_off = SHORT_A + (OP == DX ? col * 128 + (((lane >> 5) ^ ((col >> 1) & 7)) << 4) : quarter_tr_off(wave >> 1, (wave & 1) * 32, lane));
  f32x16 acc[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
#pragma unroll
  for (int q = 0; q < SHORT_DEPTH; ++q)
    if (kt0 + q < kt1) issue(kt0 + q, q);
  int slot = 0;
  for (int kt = kt0; kt < kt1; ++kt) {
    if (kt + 2 < kt1) asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
    else if (kt + 1 < kt1) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    const char* st = lds + slot * SHORT_STAGE;
    bf16x8 fa[4][2], fb[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      fb[s] = OP == DX ? lds_frag_kc(st + (b_off ^ (s * 32))) : quarter_frag_tr(st + b_off + s * 2048);
#pragma unroll
      for (int i = 0; i < 2; ++i) fa[s][i] = lds_frag_kc(st + (a_off[i] ^ (s * 32)));
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();                  // every wavefront has its fragments: the stage is free
    if (kt + SHORT_DEPTH < kt1) issue(kt + SHORT_DEPTH, slot);
    slot = slot == SHORT_DEPTH - 1 ? 0 : slot + 1;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if ((kt + 1) * QK > depth && kt * QK + 16 * s + 8 * (lane >> 5) >= depth) fa[s][0] = fa[s][1] = fb[s] = bf16x8{};
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[s][i], fb[s], acc[i], 0, 0, 0);
    }
  }
  float* const slab = reinterpret_cast<float*>(lds) + wave * (SHORT * SHORT_PITCH);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) slab[(32 * i + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * SHORT_PITCH + (lane & 31)] = acc[i][r];
  __builtin_amdgcn_wave_barrier();
  const int out_col = n0 + wave * 32 + (lane & 3) * 8;
  if (out_col >= p.N) return;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int in = 16 * q + (lane >> 2);
    if (in >= rows) break;
    const float* const from = slab + in * SHORT_PITCH + (lane & 3) * 8;
    store_out<OP>(l, p, t.e, p.parts.n, part, (size_t)(row0 + in) * p.N + out_col, out_col, from);
  }
}

// STREAM (FWD, DX): weights that one tile reads are loaded as such
template <int OP, bool STREAM = false>
__device__ __forceinline__ void multiply_tile(const LinearArgs& l, const Product& p, int b, int part, char* lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  Tile t;
  if (!tile_of<OP>(l, p, b, part, lane, t)) return;
  if constexpr (OP != DW)
    if (t.end - t.first <= SHORT) return multiply_short<OP, STREAM>(l, p, t, part, lds);
  const int n0 = t.nt * QT;
  const int row0 = OP == DW ? t.mt * QT : t.first + t.mt * QT, row_end = OP == DW ? p.M : t.end;      // of the output
  // k-tiles [kt, kt1) of 64, of the whole contraction [0, depth)
  const int depth = OP == DW ? t.end - t.first : p.K, parts = OP == DW ? parts_of_expert<bf16_t>(l.offsets, depth, p.parts.n) : p.parts.n;
  if (OP == DW && part >= parts) return;
  const int all = (depth + QK - 1) / QK, per = (all + parts - 1) / parts, kt0 = min(all, part * per), kt1 = min(all, kt0 + per);

  const uint32_t base = lds_addr(lds);
  QuarterKc a_kc, b_kc;
  QuarterTr a_tr, b_tr;
  if (OP == DW) {
    a_tr.setup(p.A + (size_t)t.first * p.lda, nullptr, false, p.lda, row0, p.M, wave, lane);
    b_tr.setup(p.B + (size_t)t.first * p.ldb, nullptr, false, p.ldb, n0, p.N, wave, lane);
  } else {
    a_kc.setup(p.A + (size_t)row0 * p.lda, p.lda, row_end - row0, wave, lane);
    if (OP == FWD) b_tr.setup(p.B + (size_t)t.e * p.b_es, nullptr, false, p.ldb, n0, p.N, wave, lane);
    else b_kc.setup(p.B + (size_t)t.e * p.b_es + (size_t)n0 * p.ldb, p.ldb, p.N - n0, wave, lane);
  }
  auto issue = [&](int kt) {
    const uint32_t st = base + (kt & 1) * STAGE;
    const long k0 = (long)kt * QK;
    const int last = depth - 1 - (int)k0;          // >= 0
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t back = OP != DW && last < QK - 1 ? past_end((int)k0 + 8 * QuarterKc::chunk(j, lane), depth) : 0;
      if (OP == DW) a_tr.template issue1<true>(j, st, wave, lane, k0, last);
      else a_kc.issue1(j, st, wave, k0, back);
      if (OP == DX) b_kc.template issue1<STREAM>(j, st + QOPER_BYTES, wave, k0, back);
      else b_tr.template issue1<true, STREAM>(j, st + QOPER_BYTES, wave, lane, k0, last);
    }
  };
  int a_off[2], b_off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = wm * 64 + i * 32 + (lane & 31), col = wn * 64 + i * 32 + (lane & 31);
    a_off[i] = OP == DW ? quarter_tr_off(wm, i * 32, lane) : row * 128 + (((lane >> 5) ^ ((row >> 1) & 7)) << 4);
    b_off[i] = QOPER_BYTES + (OP == DX ? col * 128 + (((lane >> 5) ^ ((col >> 1) & 7)) << 4) : quarter_tr_off(wn, i * 32, lane));
  }
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  if (kt0 < kt1) issue(kt0);
  if (kt0 + 1 < kt1) issue(kt0 + 1);
  for (int kt = kt0; kt < kt1; ++kt) {
    if (kt + 1 < kt1) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    const char* st = lds + (kt & 1) * STAGE;
    bf16x8 fa[4][2], fb[4][2];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[s][i] = OP == DW ? quarter_frag_tr(st + a_off[i] + s * 2048) : lds_frag_kc(st + (a_off[i] ^ (s * 32)));
        fb[s][i] = OP == DX ? lds_frag_kc(st + (b_off[i] ^ (s * 32))) : quarter_frag_tr(st + b_off[i] + s * 2048);
      }
    if ((kt + 1) * QK > depth) {                   // zeros past the contraction's end, in both operands: either may be no number there
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int k = kt * QK + 16 * s + 8 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (OP == DW) {                          // (the rows of an expert end anywhere)
            s16x8 u = __builtin_bit_cast(s16x8, fa[s][i]), v = __builtin_bit_cast(s16x8, fb[s][i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) { u[j] = k + j < depth ? u[j] : (short)0; v[j] = k + j < depth ? v[j] : (short)0; }
            fa[s][i] = __builtin_bit_cast(bf16x8, u);
            fb[s][i] = __builtin_bit_cast(bf16x8, v);
          } else if (k >= depth) {
            fa[s][i] = fb[s][i] = bf16x8{};
          }
        }
      }
    }
    const auto step = [&](int s) {                 // blocks (0,0), (0,1), (1,1), (1,0)
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const int i = m >> 1, j = i ^ (m & 1);
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[s][i], fb[s][j], acc[i][j], 0, 0, 0);
      }
    };
    step(0);
    step(1);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();                  // every wavefront has its fragments: the stage is free
    if (kt + 2 < kt1) issue(kt + 2);
    step(2);
    step(3);
  }
  // FWD: residual and bias are on their way while the sums change places: one load after the other behind the stores takes 8192 rows of 256 to 8192
  // with z and residual from 128 to 160 us.  (The gradients, 4096 rows of 2880 to 2880, so: 162 -> 178.)
  const int col = n0 + wn * 64 + (lane & 7) * 8, first_row = row0 + wm * 64 + (lane >> 3);
  const auto at_row = [&](int row) { return ((size_t)(OP == DW ? t.e : 0) * p.M + row) * p.N + col; };
  const bf16_t* const old = parts > 1 ? nullptr : (const bf16_t*)l.residual;
  u32x4 pre[8];
  float bias[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) bias[j] = 0.f;
  if (OP == FWD && col < p.N) {
    if (parts == 1 && l.bias) values(*reinterpret_cast<const u32x4*>((const bf16_t*)l.bias + (size_t)t.e * l.N + col), bias);
    if (old)
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (first_row + 8 * q < row_end) pre[q] = *reinterpret_cast<const u32x4*>(old + at_row(first_row + 8 * q));
  }
  // Element 4 g + q of a lane's block is row 8 g + 4 (lane / 32) + q, column lane % 32: through the wavefront's own slab to eight columns a lane.
  float* const slab = reinterpret_cast<float*>(lds) + wave * (SLAB / 4);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        slab[(32 * i + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * TILE_PITCH + 32 * j + (lane & 31)] = acc[i][j][r];
  __builtin_amdgcn_wave_barrier();
  if (col >= p.N) return;
  if constexpr (OP == FWD) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int row = first_row + 8 * q;
      if (row >= row_end) break;
      const float* const from = slab + (8 * q + (lane >> 3)) * TILE_PITCH + (lane & 7) * 8;
      if (parts > 1) {
        store_out<OP>(l, p, t.e, parts, part, at_row(row), col, from);
        continue;
      }
      float y[8], add[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = from[j] + bias[j];
      activate_forward<bf16_t>(l, at_row(row), y);
      if (old) {
        values(pre[q], add);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] += add[j];
      }
      store_to<bf16_t>(l.y, at_row(row), y);
    }
  } else {
#pragma unroll 2
    for (int q = 0; q < 8; ++q) {
      const int row = first_row + 8 * q;
      if (row >= row_end) break;
      store_out<OP>(l, p, t.e, parts, part, at_row(row), col, slab + (8 * q + (lane >> 3)) * TILE_PITCH + (lane & 7) * 8);
    }
  }
}

// dW where the experts have few rows, bound by writing it: every wavefront forms 64 x 128 of a matrix by itself, 32 rows at a time, both operands through
// registers (linear_piece.h).  Element r of acc[i][j] is row 4 (4 (lane / 16) + r) + i, column 8 (lane % 16) + j.
constexpr int OUTER_M = 64, OUTER_N = 128, OUTER_ROWS = 64;
__device__ __forceinline__ void outer_tile(const LinearArgs& l, const Product& p, int b) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const int mt = (p.M + OUTER_M - 1) / OUTER_M, nt = (p.N + OUTER_N - 1) / OUTER_N, at = b * (NT / WAVE) + wave;
  if (at >= l.e_cnt * mt * nt) return;
  const int e = at / (mt * nt), in_e = at - e * mt * nt, m0 = in_e / nt * OUTER_M, n0 = in_e % nt * OUTER_N;
  const int first = __builtin_amdgcn_readfirstlane(l.offsets ? l.offsets[e] : 0), end = __builtin_amdgcn_readfirstlane(l.offsets ? l.offsets[e + 1] : l.rows);
  const int xcol = 2 * min(4 * i, p.M - m0 - 4), zcol = 2 * min(8 * i, p.N - n0 - 8);        // columns past the end repeat the last ones
  const int xrow = 2 * (int)p.lda, zrow = 2 * (int)p.ldb;
  f32x4 acc[4][8];
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[a][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int row = first; row < end; row += 32) {
    ColumnPiece<4> x;
    ColumnPiece<8> z;
    const bf16_t* const xb = p.A + (size_t)row * p.lda + m0;
    const bf16_t* const zb = p.B + (size_t)row * p.ldb + n0;
    if (end - row >= 32) {
      x.load<false>(xb, true, xrow, 8 * g * xrow + xcol);
      z.load<false>(zb, true, zrow, 8 * g * zrow + zcol);
    } else {
      x.load_end(xb, xrow, 8 * g, end - row, xcol);
      z.load_end(zb, zrow, 8 * g, end - row, zcol);
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const bf16x8 f = z.operand(c);
#pragma unroll
      for (int a = 0; a < 4; ++a) acc[a][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.operand(a), f, acc[a][c], 0, 0, 0);
    }
  }
  const int col = n0 + 8 * i;
  if (col >= p.N) return;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int m = m0 + 4 * (4 * g + r) + a;
      if (m >= p.M) continue;
      float y[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) y[c] = acc[a][c][r];
      finish<DW>(l, p, e, ((size_t)e * p.M + m) * p.N + col, col, y);
    }
}

template <int OP, bool STREAM = false>
__global__ __launch_bounds__(NT, 2) void linear_tiles(TileArgs a) {
  __shared__ __align__(1024) char lds[TILE_LDS];
  multiply_tile<OP, STREAM>(a.l, a.p, blockIdx.x, blockIdx.y, lds);
}

// The gradients in one launch: dW's blocks and dx's, the longer ones first, and db's.  (dx_blocks, dw_blocks: of one part; multiples of 8)
struct Gradients {
  LinearArgs l;
  Product dx, dw;
  BiasGrad db;
  int dx_blocks, dw_blocks, dx_total, dw_total;
  int outer;               // dW by outer_tile
  int dx_first;
};
template <bool STREAM>
__global__ __launch_bounds__(NT, 2) void linear_gradients(Gradients g) {
  __shared__ __align__(1024) char lds[TILE_LDS];
  int b = blockIdx.x;
  const int dw = g.dx_first ? b - g.dx_total : b, dx = g.dx_first ? b : b - g.dw_total;
  if (dx >= 0 && dx < g.dx_total) return multiply_tile<DX, STREAM>(g.l, g.dx, dx % g.dx_blocks, dx / g.dx_blocks, lds);
  if (dw >= 0 && dw < g.dw_total) {
    if (g.outer) return outer_tile(g.l, g.dw, dw);
    return multiply_tile<DW>(g.l, g.dw, dw % g.dw_blocks, dw / g.dw_blocks, lds);
  }
  b -= g.dx_total + g.dw_total;
  bias_columns<bf16_t>(g.db, b, reinterpret_cast<float*>(lds));
}
static_assert(NT == BIAS_THREADS, "");

// Time in us of a k-tile on a CU: one workgroup alone, two beside each other (both of them), and of each of many when the whole chip multiplies.
// Operands that come from memory and not from the caches take longer.
struct KTile { float alone, two, many; };
constexpr KTile CACHED = {0.58f, 0.82f, 0.56f}, STREAMED = {0.72f, 1.3f, 0.65f};
inline float k_tile(const KTile& k, float per_cu) {
  const float least = per_cu <= 1.f ? k.alone : k.two;
  return per_cu * k.many > least ? per_cu * k.many : least;
}
inline long long most_parts(long long tiles, long long k_tiles) {
  const long long parts = tiles > 0 ? CUT_WORKGROUPS / tiles : 1, deep = k_tiles / 2;
  return parts < 1 || deep < 1 ? 1 : parts > MOST_PARTS ? (deep < MOST_PARTS ? deep : MOST_PARTS) : parts < deep ? parts : deep;
}
// The forward's parts, and its time
inline float forward_time(long long tiles, long long k_tiles, double outputs, const KTile& k, int* parts) {
  float best = 0.f;
  for (int p = 1; p <= most_parts(tiles, k_tiles); ++p) {
    const float t = 6.f + (float)((k_tiles + p - 1) / p) * k_tile(k, (float)(tiles * p) / 256.f) + join_time(p, outputs);
    if (p == 1 || t < best) { best = t; *parts = p; }
  }
  return best;
}
// Parts of both gradients' products in one launch: as many as bring either's longest tile down to what the chip takes for all of them.  CACHED for every
// layer: where the weights come from memory the time is less than it takes.  us, by this model / measured: 4096 rows of 2880 to 2880 153 / 155, 1024 of
// 4096 to 4096 78 / 82, of 4096 to 14336 257 / 268; 16 experts' 32 rows of 2880 to 2880 73 / 126, 128 rows 113 / 172, 256 rows 186 / 228, 32 experts' 8
// rows of 7168 to 2048 219 / 347.
inline int chain_parts(long long tiles, long long k_tiles, float all) {
  const long long most = most_parts(tiles, k_tiles);
  const float goal = all > 5.f ? all : 5.f;
  long long p = 1;
  while (p < most && (float)((k_tiles + p - 1) / p) * CACHED.alone > goal) ++p;
  return (int)p;
}
inline long long row_tiles(const LinearArgs& l) {
  return ((long long)l.rows + QT - 1) / QT + (l.offsets ? (l.e_cnt < l.rows ? l.e_cnt : l.rows) - 1 : 0);
}
inline long long column_tiles(int n) { return (n + QT - 1) / QT; }
inline unsigned blocks_of(long long tiles) { return (unsigned)((tiles + 7) / 8 * 8); }

// No empty part: as many as parts of the rounded-up length need
inline int whole_parts(int parts, long long k_tiles) {
  const long long per = (k_tiles + parts - 1) / parts;
  return per > 0 ? (int)((k_tiles + per - 1) / per) : 1;
}
// whether the forward's weights come from memory: those of one layer, beyond what the Infinity Cache may keep of them
inline bool streamed(const LinearArgs& l) { return 2ll * l.K * l.N * l.e_cnt > (100ll << 20); }
Product forward_of(const LinearArgs& l, void* ws, float* time) {
  Product p = {(const bf16_t*)l.x, (const bf16_t*)l.w, l.K, l.N, (long)l.K * l.N, (bf16_t*)l.y, 0, l.N, l.K, {(float*)ws, (size_t)l.rows * l.N, 1}, 0};
  p.tiles = row_tiles(l) * column_tiles(l.N);
  const long long k_tiles = (l.K + QK - 1) / QK;
  *time = forward_time(p.tiles, k_tiles, (double)l.rows * l.N, streamed(l) ? STREAMED : CACHED, &p.parts.n);
  p.parts.n = whole_parts(p.parts.n, k_tiles);
  return p;
}
Product dx_of(const LinearArgs& l, const void* dz, void* dx, int accumulate, void* ws) {
  Product p = {(const bf16_t*)dz, (const bf16_t*)l.w, l.N, l.N, (long)l.K * l.N, (bf16_t*)dx, 0, l.K, l.N, {(float*)ws, (size_t)l.rows * l.K, 1}, accumulate};
  p.tiles = row_tiles(l) * column_tiles(l.K);
  return p;
}
Product dw_of(const LinearArgs& l, const void* dz, void* dw, int accumulate, void* ws) {
  Product p = {(const bf16_t*)l.x, (const bf16_t*)dz, l.K, l.N, 0, (bf16_t*)dw, l.K, l.N, 0, {(float*)ws, (size_t)l.e_cnt * l.K * l.N, 1}, accumulate};
  p.tiles = l.e_cnt * column_tiles(l.K) * column_tiles(l.N);
  return p;
}
inline long long outer_waves(const LinearArgs& l) {
  return (long long)l.e_cnt * ((l.K + OUTER_M - 1) / OUTER_M) * ((l.N + OUTER_N - 1) / OUTER_N);
}
// parts of both; returns the time of their launch and of the one that adds the parts up
float plan_gradients(const LinearArgs& l, Product& x, Product& w, bool* outer, bool* dx_first) {
  const long long kx = (l.N + QK - 1) / QK, kw = ((long long)l.rows / l.e_cnt + QK - 1) / QK;
  *outer = w.C && (long long)OUTER_ROWS * l.e_cnt >= l.rows;
  const float all = CACHED.many / 256.f * (float)((x.C ? x.tiles * kx : 0) + (w.C && !*outer ? w.tiles * kw : 0)) +
                    (*outer ? (float)outer_waves(l) * (1.5f / 2048.f) * (float)(1 + (l.rows / l.e_cnt + 31) / 32) : 0.f);
  float chain = 0.f, join = 0.f;
  *dx_first = true;
  double parts = 0;
  if (x.C) {
    x.parts.n = whole_parts(chain_parts(x.tiles, kx, all), kx);
    chain = (float)((kx + x.parts.n - 1) / x.parts.n) * CACHED.alone;
    if (x.parts.n > 1) { join = 3.f; parts += (double)x.parts.n * l.rows * l.K; }
  }
  if (w.C && !*outer) {
    w.parts.n = chain_parts(w.tiles, kw, all);
    // experts whose rows differ: parts, where one of six times the mean rows would take 14 us longer than all of them otherwise
    const long long longest = (longest_rows(l) + QK - 1) / QK;
    if (l.offsets && (float)longest * CACHED.alone > all + 14.f) w.parts.n = (int)most_parts(w.tiles, longest);
    const int mean_parts = l.offsets ? (int)std::max(1ll, std::min<long long>(w.parts.n, kw / 8)) : w.parts.n;
    const float c = (float)((kw + mean_parts - 1) / mean_parts) * CACHED.alone;
    *dx_first = chain >= c;
    chain = c > chain ? c : chain;
    if (w.parts.n > 1) { join = 3.f; parts += (double)mean_parts * l.e_cnt * l.K * l.N; }
  }
  return 6.f + (all > chain ? all : chain) + join + (float)(parts * (8.0 / 9e6));
}

}  // namespace

// Sums of parts of an output of `rows` x `columns`, for any number of rows up to this one: at most MOST_PARTS times the output, and CUT_WORKGROUPS tiles
size_t linear_parts_bytes(long long rows, int columns) {
  const size_t all = (size_t)MOST_PARTS * rows * columns * 4, most = (size_t)CUT_WORKGROUPS * QT * QT * 4;
  return all < most ? all : most;
}

float linear_tiles_fwd_time(const LinearArgs& l) {
  float t;
  forward_of(l, nullptr, &t);
  return t;
}
float linear_tiles_bwd_time(const LinearArgs& l, bool dx, bool dw) {
  void* const some = (void*)1;
  Product x = dx_of(l, nullptr, dx && l.rows > 0 ? some : nullptr, 0, nullptr), w = dw_of(l, nullptr, dw ? some : nullptr, 0, nullptr);
  bool outer, dx_first;
  return plan_gradients(l, x, w, &outer, &dx_first);
}

int launch_linear_tiles_fwd(const LinearArgs& l, void* ws, hipStream_t s) {
  float time;
  const TileArgs a = {l, forward_of(l, ws, &time)};
  const unsigned blocks = blocks_of(a.p.tiles);
  ProfScope prof(MOE_K_LINEAR, s);
  // (stream_rule.h: weights that one tile reads and that the Infinity Cache does not keep)
  if (l.rows <= (long long)QT * l.e_cnt && 2ll * l.K * l.N * l.e_cnt > (256ll << 20)) hipLaunchKernelGGL((linear_tiles<FWD, true>), dim3(blocks, a.p.parts.n), dim3(NT), 0, s, a);
  else hipLaunchKernelGGL(linear_tiles<FWD>, dim3(blocks, a.p.parts.n), dim3(NT), 0, s, a);
  HIP_CHECK_LAUNCH();
  return launch_join_forward<bf16_t>(l, a.p.parts, s);
}

// ws_dx: linear_parts_bytes(rows, K), ws_dw: linear_parts_bytes(e_cnt * K, N)
int launch_linear_tiles_bwd(const LinearArgs& l, const void* dz, void* dx, int dx_accumulate, void* dw, int accumulate, const BiasGrad& db, void* ws_dx, void* ws_dw,
                            hipStream_t s) {
  Product x = dx_of(l, dz, l.rows > 0 ? dx : nullptr, dx_accumulate, ws_dx), w = dw_of(l, dz, dw, accumulate, ws_dw);
  bool outer, dx_first;
  plan_gradients(l, x, w, &outer, &dx_first);
  Gradients g = {l, x, w, db, (int)blocks_of(x.tiles), l.offsets ? (int)((w.tiles + 255) / 256 * 256) : (int)blocks_of(w.tiles), 0, 0, outer, dx_first};
  if (x.C) g.dx_total = g.dx_blocks * x.parts.n;
  if (w.C) g.dw_total = outer ? (int)((outer_waves(l) + 3) / 4) : g.dw_blocks * w.parts.n;
  const unsigned blocks = g.dx_total + g.dw_total + (db.db ? bias_blocks(l.N, l.e_cnt) : 0);
  if (blocks > 0) {
    ProfScope prof(x.C && w.C ? MOE_K_LINEAR_DX_DW : w.C ? MOE_K_LINEAR_DW : x.C ? MOE_K_LINEAR_DX : MOE_K_LINEAR_BIAS, s);
    const bool stream = l.rows <= (long long)QT * l.e_cnt && 2ll * l.K * l.N * l.e_cnt > (256ll << 20);
    hipLaunchKernelGGL(stream ? linear_gradients<true> : linear_gradients<false>, dim3(blocks), dim3(NT), 0, s, g);
    HIP_CHECK_LAUNCH();
  }
  return launch_join_gradients<bf16_t>(l, x.parts, dx, dx_accumulate, w.parts, dw, accumulate, s);
}
