// The experts' forward in microscaled 4 bits (mx4.h): rows, weights and activations are e2m1 with a scale per 32 elements, the products run on
// the scaled matrix instruction, sums are fp32.
//
//   rows    xq = MX4(xp)                                  every expert's rows begin at a tile of 16
//   UP      aq = MX4(silu(xq W1) * (xq W3))
//   DOWN    o  = aq W2                                    bf16
#include "mx4.h"
#include "kernels.h"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

enum { UP, DOWN };

struct XArgs {
  const uint8_t* A; const uint8_t* As;         // rows: tiles of 16, an expert's from first[e] on
  const uint8_t* B0; const uint8_t* Bs0;       // weights
  const uint8_t* B1; const uint8_t* Bs1;       // UP: W3
  size_t b_es, bs_es;                          // bytes from an expert's to the next one's
  uint8_t* C; uint8_t* Cs;                     // UP: aq
  bf16_t* O;                                   // DOWN
  const int32_t* off; const int32_t* first;
  int e_cnt, N, K;
};

// element r of the 16x16 result in a lane: weight column 4 (lane / 16) + r, row lane % 16
template <int SA, int SB>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c, uint32_t sa, uint32_t sb) {
  const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, SA, (int)sa, SB, (int)sb);      // 4: e2m1
}

// ---- rows: 16 rows by 512 elements per wavefront, as mx4_rows; a block finds its tile's expert by itself
constexpr int ROWS_BLOCK = 256;
__global__ __launch_bounds__(ROWS_BLOCK) void expert_rows(const bf16_t* __restrict__ x, const int32_t* __restrict__ off, int e_cnt, int d, int f,
                                                           uint8_t* __restrict__ q, uint8_t* __restrict__ scales, uint8_t* __restrict__ aq,
                                                           uint8_t* __restrict__ as, int32_t* __restrict__ first) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = blockIdx.x, group = blockIdx.y * (ROWS_BLOCK / WAVE) + wave;
  int e = -1, row_tile = 0, before = 0;
  const bool writes = blockIdx.x == 0 && blockIdx.y == 0 && wave == 0;
  for (int base = 0; base < e_cnt; base += WAVE) {
    const int i = base + lane, n = i < e_cnt ? (off[i + 1] - off[i] + 15) / 16 : 0, incl = wave_scan(n);
    if (writes && i < e_cnt) first[i] = before + incl - n;
    const unsigned long long past = __ballot(before + incl > tile);
    if (e < 0 && past) {
      const int who = __builtin_ctzll(past);
      e = base + who;
      row_tile = tile - before - __builtin_amdgcn_readlane(incl - n, who);
      if (!writes) break;
    }
    before += __builtin_amdgcn_readlane(incl, WAVE - 1);
  }
  const int groups = mx_groups(d), depths = mx_depths(d);
  if (e < 0 || group >= groups) return;
  const int row = off[e] + 16 * row_tile + (lane & 15), chunk = lane >> 4;
  const bool in = row < off[e + 1];
  const bf16_t* src = x + (size_t)row * d;
  uint32_t word = 0;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int depth = 4 * group + p, k = MX_DEPTH * depth + MX_CHUNK * chunk;
    if (depth >= depths) break;
    uint32_t byte = 0;
    mx_u32x4 codes = {0, 0, 0, 0};
    if (in && k < d) codes = mx_load_chunk(src + k, byte);
    word |= byte << (8 * p);
    *reinterpret_cast<mx_u32x4*>(q + ((size_t)tile * depths + depth) * MX_TILE + lane * 16) = codes;
  }
  *reinterpret_cast<uint32_t*>(scales + ((size_t)tile * groups + group) * MX_SCALES + lane * 4) = word;
  // the chunks of the activations past f, which UP does not write
  if (group == 0 && f % MX_DEPTH != 0 && chunk >= f % MX_DEPTH / MX_CHUNK) {
    const int depth = f / MX_DEPTH;
    *reinterpret_cast<mx_u32x4*>(aq + ((size_t)tile * mx_depths(f) + depth) * MX_TILE + lane * 16) = mx_u32x4{0, 0, 0, 0};
    as[((size_t)tile * mx_groups(f) + depth / 4) * MX_SCALES + lane * 4 + depth % 4] = 0;
  }
}

// ---- a few rows per expert: up to 16 * TG rows against 32 columns (UP: 32 of either matrix).  The wavefronts of a block share the contraction,
// wavefront w the pieces w, w + NW, .. of 512, and their sums are added in LDS in ascending order.
constexpr int FEW_ROWS = 32, FEW_WAVES = 8, FEW_COLS = 32;
template <int MODE, int TG>
__device__ __forceinline__ void few_tile(const XArgs& p, f32x4* lds, int e, int row_tile, int n0, int rows) {
  constexpr int NB = MODE == UP ? 4 : 2;       // 16-column operands: W1's two, then W3's
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int depths = mx_depths(p.K), groups = mx_groups(p.K);
  const int tile0 = p.first[e] + row_tile * (FEW_ROWS / 16);
  f32x4 acc[NB][TG];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int t = 0; t < TG; ++t) acc[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int group = wave; group < groups; group += waves) {
    u32x4 b[NB][4], a[TG][4];
    uint32_t bs[NB], as[TG];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int nt = n0 / 16 + (j & 1);
      const uint8_t* data = (j < 2 ? p.B0 : p.B1) + e * p.b_es + (size_t)nt * depths * MX_TILE + lane * 16;
      const uint8_t* scale = (j < 2 ? p.Bs0 : p.Bs1) + e * p.bs_es + ((size_t)nt * groups + group) * MX_SCALES + lane * 4;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        b[j][q] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(data + (size_t)min(4 * group + q, depths - 1) * MX_TILE));
      bs[j] = *reinterpret_cast<const uint32_t*>(scale);
    }
#pragma unroll
    for (int t = 0; t < TG; ++t) {
      const uint8_t* data = p.A + (size_t)(tile0 + t) * depths * MX_TILE + lane * 16;
#pragma unroll
      for (int q = 0; q < 4; ++q) a[t][q] = *reinterpret_cast<const u32x4*>(data + (size_t)min(4 * group + q, depths - 1) * MX_TILE);
      as[t] = *reinterpret_cast<const uint32_t*>(p.As + ((size_t)(tile0 + t) * groups + group) * MX_SCALES + lane * 4);
    }
    static_for<4>([&](auto at) {
      constexpr int q = decltype(at)::value;
      if (4 * group + q < depths) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int t = 0; t < TG; ++t) acc[j][t] = mfma<q, q>(b[j][q], a[t][q], acc[j][t], bs[j], as[t]);
      }
    });
  }
  const int i = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < TG; ++t) {
    if (waves > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NB; ++j) lds[(wave * NB + j) * WAVE + lane] = acc[j][t];
      __syncthreads();
    }
    if (wave != t % waves) continue;
    f32x4 sum[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      sum[j] = acc[j][t];
      if (waves > 1) {
        sum[j] = lds[j * WAVE + lane];
        for (int w = 1; w < waves; ++w) sum[j] += lds[(w * NB + j) * WAVE + lane];
      }
    }
    if constexpr (MODE == UP) {
      // this lane's eight of the row's 32 activations: columns 16 j + 4 g + r
      float v[2][4];
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          v[j][r] = silu_f(sum[j][r]) * sum[2 + j][r];
          top = max(top, __float_as_uint(v[j][r]) & 0x7FFFFFFFu);
        }
      top = max(top, (uint32_t)__shfl_xor((int)top, 16));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      const uint32_t byte = mx_scale_byte(top);
      const float s = mx_scale_value(byte);
      uint32_t codes = 0;
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[0][0], v[0][1], s, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[0][2], v[0][3], s, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[1][0], v[1][1], s, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[1][2], v[1][3], s, 3);
      if (byte == 255) codes = 0;
      const int depth = n0 / MX_DEPTH, chunk = n0 % MX_DEPTH / MX_CHUNK;
      uint16_t* out = reinterpret_cast<uint16_t*>(p.C + ((size_t)(tile0 + t) * mx_depths(p.N) + depth) * MX_TILE + chunk * 256 + i * 16);
      out[g] = (uint16_t)codes;
      out[4 + g] = (uint16_t)(codes >> 16);
      if (g == 0) p.Cs[((size_t)(tile0 + t) * mx_groups(p.N) + depth / 4) * MX_SCALES + chunk * 64 + i * 4 + depth % 4] = (uint8_t)byte;
    } else if (16 * t + i < rows) {
      bf16_t* out = p.O + ((size_t)p.off[e] + row_tile * FEW_ROWS + 16 * t + i) * p.N + n0 + 4 * g;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        *reinterpret_cast<u32x2*>(out + 16 * j) = u32x2{pack_bf16x2(sum[j][0], sum[j][1]), pack_bf16x2(sum[j][2], sum[j][3])};
    }
  }
}

// Experts in the order of RaggedTiles, but only those whose row count lies in (LO, hi]; rows in tiles of TM.
template <int TM>
struct SomeTiles {
  const int32_t* off;
  int e_cnt, lane, lo, hi;
  int n, incl, total;
  __device__ __forceinline__ int count(int e) const {
    const int rows = e < e_cnt ? off[e + 1] - off[e] : 0;
    return rows > lo && rows <= hi ? (rows + TM - 1) / TM : 0;
  }
  __device__ __forceinline__ SomeTiles(const int32_t* __restrict__ off_, int e_cnt_, int lane_, int lo_, int hi_)
      : off(off_), e_cnt(e_cnt_), lane(lane_), lo(lo_), hi(hi_) {
    n = count(lane);
    incl = wave_scan(n);
    total = __builtin_amdgcn_readlane(incl, WAVE - 1);
    for (int base = WAVE; base < e_cnt; base += WAVE) total += wave_sum(count(base + lane));
  }
  // tile b of a walk that goes through every XCD's contiguous eighth; false: past its end
  __device__ __forceinline__ bool tile(int n_cols, int b, int& e, int& row_tile, int& col_tile) const {
    const int share = (total * n_cols + 7) / 8;
    const int at = (b % 8) * share + b / 8;
    if (b / 8 >= share || at >= total * n_cols) return false;
    int t = at / n_cols, rows = n, up_to = incl;
    col_tile = at - t * n_cols;
    for (int base = 0;; base += WAVE) {          // ends: t < total
      if (base > 0) up_to = wave_scan(rows = count(base + lane));
      const unsigned long long past = __ballot(up_to > t);
      if (past) {
        const int who = __builtin_ctzll(past);
        row_tile = t - __builtin_amdgcn_readlane(up_to - rows, who);
        e = base + who;
        return true;
      }
      t -= __builtin_amdgcn_readlane(up_to, WAVE - 1);
    }
  }
};

template <int MODE>
__global__ __launch_bounds__(FEW_WAVES * WAVE) void few_rows_mx4(XArgs p) {
  __shared__ f32x4 lds[FEW_WAVES * (MODE == UP ? 4 : 2) * WAVE];
  const SomeTiles<FEW_ROWS> list(p.off, p.e_cnt, threadIdx.x & 63, 0, 0x7FFFFFFF);
  int e, row_tile, col_tile;
  if (!list.tile(p.N / FEW_COLS, blockIdx.x, e, row_tile, col_tile)) return;
  const int rows = p.off[e + 1] - p.off[e] - row_tile * FEW_ROWS;
  if (rows <= 16) few_tile<MODE, 1>(p, lds, e, row_tile, col_tile * FEW_COLS, rows);
  else few_tile<MODE, 2>(p, lds, e, row_tile, col_tile * FEW_COLS, rows);
}

// ---- many rows per expert: 128 rows against 256 weight rows (UP: 128 of either matrix), four wavefronts of 64 by 128 in 32x32x64
// instructions.  Operands go from memory to LDS directly, 128 of the contraction at a time through a ring of three stages; their layout in
// memory is the one that the instruction wants, so every load is 1 KB of consecutive bytes and every LDS read free of conflicts.
constexpr int GEMM_ROWS = 128, GEMM_COLS = 256, GEMM_THREADS = 256;
constexpr int STAGE_TILES = (GEMM_ROWS + GEMM_COLS) / 16, STAGE = STAGE_TILES * MX_TILE, STAGES = 3;
constexpr int STAGE_LOADS = STAGE_TILES / 4, SCALE_LOADS = 2;           // per wavefront
constexpr int GEMM_LDS = STAGES * STAGE + STAGE_TILES * MX_SCALES;
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int S>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c, uint32_t sa, uint32_t sb) {
  const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, S, (int)sa, S, (int)sb);
}
// lanes 32..63 of a and lanes 0..31 of b change places
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
template <int N>
__device__ __forceinline__ void wait_and_meet() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory"); }

template <int MODE>
__device__ __forceinline__ void gemm_tile(const XArgs& p, uint8_t* lds, int e, int row_tile, int col_tile, int rows) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int depths = mx_depths(p.K), groups = mx_groups(p.K);
  const int tile0 = p.first[e] + row_tile * (GEMM_ROWS / 16), row_tiles = (min(rows, GEMM_ROWS) + 15) / 16;
  const int cols = MODE == UP ? GEMM_COLS / 2 : GEMM_COLS, n0 = col_tile * cols, col_tiles = min(cols, p.N - n0) / 16;
  const uint32_t lds0 = lds_addr(lds), scales0 = lds0 + STAGES * STAGE;
  // Operand tile i of a stage: 0..7 the rows', 8..23 the weights' (UP: 8 of W1, 8 of W3); wavefront w loads 6 w .. 6 w + 5.  Tiles past the
  // rows or columns repeat the last one: their results are not stored.
  const uint8_t* data[STAGE_LOADS];
#pragma unroll
  for (int j = 0; j < STAGE_LOADS; ++j) {
    const int i = STAGE_LOADS * wave + j;
    const uint8_t* base;
    int t;
    if (i < 8) {
      base = p.A; t = tile0 + min(i, row_tiles - 1);
    } else {
      const int c = i - 8;
      base = (MODE == UP && c >= 8 ? p.B1 : p.B0) + e * p.b_es;
      t = n0 / 16 + min(MODE == UP ? c & 7 : c, col_tiles - 1);
    }
    data[j] = base + (size_t)t * depths * MX_TILE;
  }
  // Scales of 512: four operand tiles per load.  Of the six loads wavefront w makes the weights' w-th and the rows' w % 2-th (twice the same
  // bytes to the same place, so that all wavefronts wait for equally many).
  const uint8_t* scale_a;
  const uint8_t* scale_b;
  uint32_t voff_a, voff_b;
  {
    const int ta = 4 * (wave & 1) + lane / 16, tb = 4 * wave + lane / 16;
    scale_a = p.As + (size_t)tile0 * groups * MX_SCALES;
    voff_a = (uint32_t)(min(ta, row_tiles - 1) * groups * MX_SCALES + lane % 16 * 16);
    scale_b = (MODE == UP && wave >= 2 ? p.Bs1 : p.Bs0) + e * p.bs_es + (size_t)(n0 / 16) * groups * MX_SCALES;
    voff_b = (uint32_t)(min(MODE == UP ? tb & 7 : tb, col_tiles - 1) * groups * MX_SCALES + lane % 16 * 16);
  }
  const uint32_t voff = lane * 16;
  auto issue = [&](int t) {
    if (t % 4 == 0) {
      const size_t at = (size_t)(t / 4) * MX_SCALES;
      lds_load16((const bf16_t*)(scale_a + at), voff_a, scales0 + (wave & 1) * 1024);
      lds_load16((const bf16_t*)(scale_b + at), voff_b, scales0 + 2048 + wave * 1024);
    }
    const uint32_t slot = lds0 + t % STAGES * STAGE + STAGE_LOADS * wave * MX_TILE;
#pragma unroll
    for (int j = 0; j < STAGE_LOADS; ++j) lds_load16((const bf16_t*)(data[j] + (size_t)t * MX_TILE), voff, slot + j * MX_TILE);
  };
  const int wr = wave & 1, wc = wave >> 1, h = lane >> 5;
  const bool active = 64 * wr < rows;                 // (of a tile with up to 64 rows two wavefronts only load)
  // weights: 32-column operand j of this wavefront begins at tile b_tile(j) of the stage
  const auto b_tile = [&](int j) { return MODE == UP ? 8 + 8 * (j >> 1) + 4 * wc + 2 * (j & 1) : 8 + 8 * wc + 2 * j; };
  const int at = (lane >> 4 & 1) * MX_TILE + h * 256 + (lane & 15) * 16, scale_at = (lane >> 4 & 1) * MX_SCALES + h * 64 + (lane & 15) * 4;
  f32x16 acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  uint32_t as[2][2], bs[4][2];
  const uint8_t* const scales = lds + STAGES * STAGE + scale_at;
  __syncthreads();                                    // the stages may still be read for the tile before
  issue(0);
  if (depths > 1) issue(1);
  auto stage = [&](int t, auto which) {
    constexpr int Q = decltype(which)::value;         // t % 4
    if (t + 1 < depths) wait_and_meet<STAGE_LOADS + (Q == 3 ? SCALE_LOADS : 0)>();
    else wait_and_meet<0>();
    if (t + 2 < depths) issue(t + 2);
    if (!active) return;
    if (Q == 0) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int i = 0; i < 2; ++i) as[i][s] = *reinterpret_cast<const uint32_t*>(scales + (4 * wr + 2 * i) * MX_SCALES + 128 * s);
#pragma unroll
        for (int j = 0; j < 4; ++j) bs[j][s] = *reinterpret_cast<const uint32_t*>(scales + b_tile(j) * MX_SCALES + 128 * s);
      }
    }
    const uint8_t* const slot = lds + t % STAGES * STAGE + at;
    u32x4 a[2][2], b[2][4];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int i = 0; i < 2; ++i) a[s][i] = *reinterpret_cast<const u32x4*>(slot + (4 * wr + 2 * i) * MX_TILE + 512 * s);
#pragma unroll
      for (int j = 0; j < 4; ++j) b[s][j] = *reinterpret_cast<const u32x4*>(slot + b_tile(j) * MX_TILE + 512 * s);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = mfma32<Q>(b[s][j], a[s][i], acc[i][j], bs[j][s], as[i][s]);
  };
  for (int t = 0; t < depths; t += 4)
    static_for<4>([&](auto q) {
      if (t + decltype(q)::value < depths) stage(t + decltype(q)::value, q);
    });
  if (!active) return;
  // element 4 g + r of acc[i][j]: row lane % 32, column 8 g + 4 h + r of the 32
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 64 * wr + 32 * i + (lane & 31);
    if constexpr (MODE == UP) {
      const int tile = tile0 + row / 16;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float v[16];
        uint32_t top = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          v[r] = silu_f(acc[i][j][r]) * acc[i][j + 2][r];
          top = max(top, __float_as_uint(v[r]) & 0x7FFFFFFFu);
        }
        uint32_t other = top;
        swap32(top, other);
        const uint32_t byte = mx_scale_byte(max(top, other));
        const float s = mx_scale_value(byte);
        uint32_t lo = byte == 255 ? 0u : mx_pack8(v, s), hi = byte == 255 ? 0u : mx_pack8(v + 8, s);
        swap32(lo, hi);                               // now bytes 8 h .. 8 h + 7 of the chunk, in halves of two lanes
        const u32x2 codes = {__builtin_amdgcn_perm(hi, lo, 0x05040100u), __builtin_amdgcn_perm(hi, lo, 0x07060302u)};
        const int col = n0 + 64 * wc + 32 * j;
        if (row >= rows || col >= p.N) continue;
        const int depth = col / MX_DEPTH, chunk = col % MX_DEPTH / MX_CHUNK;
        *reinterpret_cast<u32x2*>(p.C + ((size_t)tile * mx_depths(p.N) + depth) * MX_TILE + chunk * 256 + row % 16 * 16 + 8 * h) = codes;
        if (h == 0) p.Cs[((size_t)tile * mx_groups(p.N) + depth / 4) * MX_SCALES + chunk * 64 + row % 16 * 4 + depth % 4] = (uint8_t)byte;
      }
    } else {
      bf16_t* const out = p.O + ((size_t)p.off[e] + row_tile * GEMM_ROWS + row) * p.N + n0 + 128 * wc + 16 * h;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t w[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) w[r] = pack_bf16x2(acc[i][j][2 * r], acc[i][j][2 * r + 1]);
#pragma unroll
        for (int r = 0; r < 4; ++r) swap32(w[r], w[r + 4]);         // columns 16 h .. 16 h + 15
        if (row >= rows || n0 + 128 * wc + 32 * j >= p.N) continue;
        reinterpret_cast<u32x4*>(out + 32 * j)[0] = u32x4{w[0], w[1], w[4], w[5]};
        reinterpret_cast<u32x4*>(out + 32 * j)[1] = u32x4{w[2], w[3], w[6], w[7]};
      }
    }
  }
}

// Workgroups walk the tiles of the experts with many rows, then those of the experts with few.
constexpr int FEW_MOST = 32;               // rows
template <int MODE>
__global__ __launch_bounds__(GEMM_THREADS, 2) void experts_mx4(XArgs p) {
  extern __shared__ uint8_t gemm_lds[];
  const int lane = threadIdx.x & 63;
  int e, row_tile, col_tile;
  {
    const SomeTiles<GEMM_ROWS> list(p.off, p.e_cnt, lane, FEW_MOST, 0x7FFFFFFF);
    const int cols = MODE == UP ? GEMM_COLS / 2 : GEMM_COLS;
    for (int b = blockIdx.x; list.tile((p.N + cols - 1) / cols, b, e, row_tile, col_tile); b += gridDim.x)
      gemm_tile<MODE>(p, gemm_lds, e, row_tile, col_tile, p.off[e + 1] - p.off[e] - row_tile * GEMM_ROWS);
  }
  const SomeTiles<FEW_ROWS> list(p.off, p.e_cnt, lane, 0, FEW_MOST);
  for (int b = blockIdx.x; list.tile(p.N / FEW_COLS, b, e, row_tile, col_tile); b += gridDim.x) {
    const int rows = p.off[e + 1] - p.off[e] - row_tile * FEW_ROWS;
    __syncthreads();
    if (rows <= 16) few_tile<MODE, 1>(p, reinterpret_cast<f32x4*>(gemm_lds), e, row_tile, col_tile * FEW_COLS, rows);
    else few_tile<MODE, 2>(p, reinterpret_cast<f32x4*>(gemm_lds), e, row_tile, col_tile * FEW_COLS, rows);
  }
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
// most tiles of tm rows that e_cnt experts with at most cap rows in all have
inline long long tiles_bound(int cap, int e_cnt, int tm) { return ((long long)cap + (long long)(tm - 1) * (cap < e_cnt ? cap : e_cnt)) / tm; }

struct Workspace {
  size_t first, xq, xs, aq, as, bytes;
  Workspace(int cap, int d, int f, int e_cnt) {
    const size_t tiles = (size_t)tiles_bound(cap, e_cnt, 16);
    first = 0;
    xq = align256((size_t)e_cnt * 4);
    xs = xq + tiles * mx_depths(d) * MX_TILE;
    aq = xs + tiles * mx_groups(d) * MX_SCALES;
    as = aq + tiles * mx_depths(f) * MX_TILE;
    bytes = as + tiles * mx_groups(f) * MX_SCALES;
    if (bytes < 256) bytes = 256;
  }
};

}  // namespace

size_t mx4_expert_ws_bytes(int cap, int d, int f, int e_cnt) { return align256(Workspace(cap, d, f, e_cnt).bytes); }

int launch_mx4_expert_fwd(const void* xp, int cap, int d, int f, int e_cnt, const int32_t* offsets, const uint8_t* w1, const uint8_t* s1,
                          const uint8_t* w3, const uint8_t* s3, const uint8_t* w2, const uint8_t* s2, void* o, void* ws, hipStream_t s) {
  if (cap == 0 || e_cnt == 0) return MOE_OK;
  const Workspace at(cap, d, f, e_cnt);
  uint8_t* const base = (uint8_t*)ws;
  int32_t* const first = (int32_t*)(base + at.first);
  const long long tiles = tiles_bound(cap, e_cnt, 16), few = tiles_bound(cap, e_cnt, FEW_ROWS);
  const long long up = 8 * ((few * (f / FEW_COLS) + 7) / 8), down = 8 * ((few * (d / FEW_COLS) + 7) / 8);
  if (tiles >= (1ll << 31) || up >= (1ll << 31) || down >= (1ll << 31)) return MOE_EUNSUPPORTED;
  {
    ProfScope prof(MOE_K_MX4_ROWS, s);
    const int waves = ROWS_BLOCK / WAVE;
    hipLaunchKernelGGL(expert_rows, dim3((unsigned)tiles, (mx_groups(d) + waves - 1) / waves), dim3(ROWS_BLOCK), 0, s, (const bf16_t*)xp, offsets,
                       e_cnt, d, f, base + at.xq, base + at.xs, base + at.aq, base + at.as, first);
    HIP_CHECK_LAUNCH();
  }
  const bool many = cap > FEW_MOST;            // some expert may have many rows
  if (many) {
    static bool attr_set[64] = {};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return MOE_EHIP;
    if (!attr_set[dev]) {
      if (hipFuncSetAttribute(reinterpret_cast<const void*>(&experts_mx4<UP>), hipFuncAttributeMaxDynamicSharedMemorySize, GEMM_LDS) != hipSuccess ||
          hipFuncSetAttribute(reinterpret_cast<const void*>(&experts_mx4<DOWN>), hipFuncAttributeMaxDynamicSharedMemorySize, GEMM_LDS) != hipSuccess)
        return MOE_EHIP;
      attr_set[dev] = true;
    }
  }
  const dim3 walkers(8 * ((2 * device_cu_count() + 7) / 8));       // (a walk stays in its XCD's eighth)
  XArgs p{};
  p.off = offsets; p.first = first; p.e_cnt = e_cnt;
  p.A = base + at.xq; p.As = base + at.xs;
  p.B0 = w1; p.Bs0 = s1; p.B1 = w3; p.Bs1 = s3;
  p.C = base + at.aq; p.Cs = base + at.as;
  p.N = f; p.K = d;
  p.b_es = (size_t)((f + 15) / 16) * mx_depths(d) * MX_TILE; p.bs_es = (size_t)((f + 15) / 16) * mx_groups(d) * MX_SCALES;
  {
    ProfScope prof(MOE_K_MX4_UP, s);
    if (many) hipLaunchKernelGGL(experts_mx4<UP>, walkers, dim3(GEMM_THREADS), GEMM_LDS, s, p);
    else hipLaunchKernelGGL(few_rows_mx4<UP>, dim3((unsigned)up), dim3(WAVE * min(FEW_WAVES, mx_groups(d))), 0, s, p);
    HIP_CHECK_LAUNCH();
  }
  p.A = p.C; p.As = p.Cs;
  p.B0 = w2; p.Bs0 = s2; p.B1 = nullptr; p.Bs1 = nullptr;
  p.O = (bf16_t*)o;
  p.N = d; p.K = f;
  p.b_es = (size_t)((d + 15) / 16) * mx_depths(f) * MX_TILE; p.bs_es = (size_t)((d + 15) / 16) * mx_groups(f) * MX_SCALES;
  {
    ProfScope prof(MOE_K_MX4_DOWN, s);
    if (many) hipLaunchKernelGGL(experts_mx4<DOWN>, walkers, dim3(GEMM_THREADS), GEMM_LDS, s, p);
    else hipLaunchKernelGGL(few_rows_mx4<DOWN>, dim3((unsigned)down), dim3(WAVE * min(FEW_WAVES, mx_groups(f))), 0, s, p);
    HIP_CHECK_LAUNCH();
  }
  return MOE_OK;
}
