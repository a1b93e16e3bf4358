// The experts' forward in microscaled 4 bits (mx4.h): rows, weights and activations are e2m1 with a scale per 32 elements, the products run on
// the scaled matrix instruction, sums are fp32.
//
//   rows    xq = MX4(xp)                                  every expert's rows begin at a tile of 16; in UP itself where there are few rows in all
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
  const bf16_t* X; int32_t* first_out;         // UP without expert_rows
  int few_most;                                // rows of an expert that few_tile takes
  int cached;                                  // experts whose weights fit the Infinity Cache
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }      // (the same in all lanes)

// element r of the 16x16 result in a lane: weight column 4 (lane / 16) + r, row lane % 16
template <int SA, int SB>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c, uint32_t sa, uint32_t sb) {
  const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, SA, (int)sa, SB, (int)sb);      // 4: e2m1
}

// ---- rows: a wavefront per 16 rows by 512 elements; a block finds its tile's expert by itself.  HBM bound: 16249 rows of 7168 56 us, 5.2 TB/s;
// a capacity of 131072 rows for them costs 8 us more, in blocks that find no tile.
constexpr int ROWS_BLOCK = 256;
__global__ __launch_bounds__(ROWS_BLOCK) void expert_rows(const bf16_t* __restrict__ x, const int32_t* __restrict__ off, int e_cnt, int d, int f,
                                                           uint8_t* __restrict__ q, uint8_t* __restrict__ scales, uint8_t* __restrict__ aq,
                                                           uint8_t* __restrict__ as, int32_t* __restrict__ first, int tile0) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = tile0 + blockIdx.x, group = blockIdx.y * (ROWS_BLOCK / WAVE) + wave;
  int e = -1, row_tile = 0, before = 0;
  const bool writes = tile == 0 && blockIdx.y == 0 && wave == 0;
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
  if (e < 0 || group >= mx_groups(d)) return;
  const int row0 = off[e] + 16 * row_tile, chunk = lane >> 4;
  mx_rows_512(x + (size_t)row0 * d, off[e + 1] - row0, d, (size_t)tile, group, lane, q, scales);
  // what UP does not write of the activations: chunks past f, and the scales behind them
  if (group == 0 && f % 512 != 0) {
    const int depth = f / MX_DEPTH;
    if (f % MX_DEPTH != 0 && chunk >= f % MX_DEPTH / MX_CHUNK)
      *reinterpret_cast<mx_u32x4*>(aq + ((size_t)tile * mx_depths(f) + depth) * MX_TILE + lane * 16) = mx_u32x4{0, 0, 0, 0};
    *reinterpret_cast<uint32_t*>(as + ((size_t)tile * mx_groups(f) + depth / 4) * MX_SCALES + lane * 4) = 0;
  }
}

// ---- a few rows per expert: up to 16 * TG rows against 32 columns (UP: 32 of either matrix), a stream of weights from memory to registers.  A
// piece is 512 of the contraction, 16 KB (UP) or 8 KB of weights, in two halves, of which three or two are on their way while one is
// multiplied.  2^cut wavefronts share a tile's contraction.  That number follows the tiles of all experts; a row's results must not, so that its sum
// is eight sums added in one order whatever the number.  DIRECT: rows come as bf16, a lane's 32 elements being a chunk, and become its operand in
// registers, 16 rows a tile.
// Bound by memory: the forward of a row each of 85 experts (4096 to 1536) reads 5.4 TB/s of weights, UP of 14 experts (7168 to 2048) with 208 rows 5.3.
// Tiles of up to 64 rows of this kind took 8 % longer at 31 experts with 63 rows on average than the larger tiles below.
constexpr int FEW_MOST = 32, FEW_ROWS = 32, FEW_COLS = 32, FEW_WAVES = 8;
// The pieces of a contraction belong to eight sums, piece q of `pieces` to sum 8 q / pieces.  A row's result is ((s0 + s1) + s2) + .., each sum its
// pieces in ascending order from zero.  Of 2^cut wavefronts the w-th takes the pieces from w pieces / 2^cut on, which are whole sums: as many
// pieces as another's, but for one.  Against one sum per wavefront the forward takes 1 to 3 % longer, at 54 experts (4096 to 1536) of a row or
// two 4 % (108 and 112 us); a row of one expert 5 % less.
constexpr int FEW_SUMS = 8, SUMS_LOG2 = 3;
__device__ __forceinline__ int first_piece(int w, int cut, int pieces) { return (w * pieces + (1 << cut) - 1) >> cut; }
struct Sums {                              // walks a wavefront's pieces
  int sum, rest, pieces;                   // 8 q = sum pieces + rest
  __device__ __forceinline__ Sums(int w, int cut, int pieces_) : sum(w << (SUMS_LOG2 - cut)), rest(FEW_SUMS * first_piece(w, cut, pieces_) - sum * pieces_), pieces(pieces_) {
    settle();
  }
  __device__ __forceinline__ void settle() {
    for (; rest >= pieces; rest -= pieces) ++sum;      // (a short contraction has fewer sums)
  }
  __device__ __forceinline__ bool last_piece() const { return rest + FEW_SUMS >= pieces; }
  __device__ __forceinline__ void next() { rest += FEW_SUMS; settle(); }
};
// Places in LDS for a tile's sums: the first wavefront's, which it adds up itself, in place 0; the others keep theirs apart, sum v in place
// 1 + v - 8 / 2^cut.
__host__ __device__ constexpr int few_places(int cut) { return cut == 0 ? 1 : 1 + FEW_SUMS - (FEW_SUMS >> cut); }
// (most with two wavefronts a tile: four tiles of five places)
constexpr int few_lds(int weight_operands, int row_operands) { return FEW_WAVES / 2 * few_places(1) * weight_operands * row_operands * WAVE * 16; }
// Where a tile's rows of bf16 begin, and how many there are (the others repeat the last one: their results are not used)
struct DirectRows { const bf16_t* x; int rows; };
template <int MODE, int TG, bool STREAM, bool DIRECT>
struct HalfPiece {
  static constexpr int NB = MODE == UP ? 4 : 2;       // 16-column operands: W1's two, then W3's
  u32x4 b[NB][2], a[TG][2][DIRECT ? 4 : 1];
  uint32_t bs[NB], as[TG];                            // of the whole piece
  template <int HALF>
  __device__ __forceinline__ void load(const XArgs& p, int e, int nt, int tile0, DirectRows direct, int piece, int depths, int groups, uint32_t lane) {
    int at[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) at[q] = min(4 * piece + 2 * HALF + q, depths - 1);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const uint8_t* data = (j < 2 ? p.B0 : p.B1) + e * p.b_es + (size_t)(nt + (j & 1)) * depths * MX_TILE;
      const uint8_t* scale = (j < 2 ? p.Bs0 : p.Bs1) + e * p.bs_es + ((size_t)(nt + (j & 1)) * groups + piece) * MX_SCALES;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const u32x4* from = reinterpret_cast<const u32x4*>(data + (size_t)at[q] * MX_TILE) + lane;
        b[j][q] = STREAM ? __builtin_nontemporal_load(from) : *from;
      }
      bs[j] = reinterpret_cast<const uint32_t*>(scale)[lane];
    }
#pragma unroll
    for (int t = 0; t < TG; ++t) {
      if constexpr (DIRECT) {
        const bf16_t* row = direct.x + (size_t)min(16 * t + (int)lane % 16, direct.rows - 1) * p.K;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          // (past the end the row's last chunk again, against weights that are zeros)
          const u32x4* from = reinterpret_cast<const u32x4*>(row + min(MX_DEPTH * at[q] + MX_CHUNK * ((int)lane / 16), p.K - MX_CHUNK));
#pragma unroll
          for (int i = 0; i < 4; ++i) a[t][q][i] = from[i];
        }
        continue;
      }
      const uint8_t* data = p.A + (size_t)(tile0 + t) * depths * MX_TILE;
#pragma unroll
      for (int q = 0; q < 2; ++q) a[t][q][0] = reinterpret_cast<const u32x4*>(data + (size_t)at[q] * MX_TILE)[lane];
      as[t] = reinterpret_cast<const uint32_t*>(p.As + ((size_t)(tile0 + t) * groups + piece) * MX_SCALES)[lane];
    }
    __builtin_amdgcn_sched_barrier(0);                // loads stay in order: waiting for one half must not wait for the next
  }
  template <int HALF>
  __device__ __forceinline__ void multiply(f32x4 (&acc)[NB][TG], int left) const {      // left: operands of 128 from the piece's first on
    static_for<2>([&](auto at) {
      constexpr int Q = decltype(at)::value, q = 2 * HALF + Q;
      if (q < left) {
#pragma unroll
        for (int t = 0; t < TG; ++t) {
          u32x4 rows = a[t][Q][0];
          uint32_t scales = as[t];
          if constexpr (DIRECT) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = a[t][Q][i / 4][i % 4];
            rows = mx_chunk(w, scales);
          }
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[j][t] = mfma<q, DIRECT ? 0 : q>(b[j][Q], rows, acc[j][t], bs[j], scales);
        }
      }
    });
    __builtin_amdgcn_sched_barrier(0);
  }
};

// tile in front of which the experts before e end
__device__ __forceinline__ int first_tile(const XArgs& p, int e, int lane) {
  int sum = 0;
  for (int i = lane; i < e; i += WAVE) sum += (p.off[i + 1] - p.off[i] + 15) / 16;
  return uniform(wave_sum(sum));
}

template <int MODE, int TG, bool STREAM, bool DIRECT>
__device__ __forceinline__ void few_tile(const XArgs& p, f32x4* lds, int cut, bool first, int e, int row_tile, int n0, int rows) {
  constexpr int NB = MODE == UP ? 4 : 2, TILE_ROWS = DIRECT ? 16 : FEW_ROWS;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave & ((1 << cut) - 1);
  const int depths = mx_depths(p.K), groups = mx_groups(p.K);
  const int tile0 = (DIRECT ? first_tile(p, e, lane) : uniform(p.first[e])) + row_tile * (TILE_ROWS / 16);
  const bool in = n0 < p.N;                           // (the last block of columns may be short of a wavefront's)
  constexpr bool TOTAL = MODE == DOWN || TG == 1;     // the first wavefront adds up in registers: UP has none left for 32 rows (30 spilled: 87 us
  // for 78 at 208 rows of 14 experts)
  f32x4 acc[NB][TG], total[NB][TG];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int t = 0; t < TG; ++t) acc[j][t] = total[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  // (a wavefront that has a tile alone does not wait for others, which may be at a tile of another height: everyone's places are where they are)
  constexpr int MOST_TG = DIRECT ? 1 : FEW_ROWS / 16;
  f32x4* const places = lds + (wave >> cut) * few_places(cut) * NB * MOST_TG * WAVE + lane;
  const auto at_place = [&](int place, int j, int t) -> f32x4& { return places[((place * NB + j) * TG + t) * WAVE]; };
  if (in) {
    constexpr int AHEAD = DIRECT ? 2 : TG == 1 ? 4 : 3, TURN = AHEAD == 3 ? 6 : 4;      // (register numbers and halves are those of a whole turn)
    HalfPiece<MODE, TG, STREAM, DIRECT> half[AHEAD];
    const DirectRows direct = {DIRECT ? p.X + ((size_t)p.off[e] + row_tile * TILE_ROWS) * p.K : nullptr, min(rows, TILE_ROWS)};
    const int piece0 = first_piece(part, cut, groups), halves = 2 * (first_piece(part + 1, cut, groups) - piece0);
    Sums sums(part, cut, groups);
    bool may_write = cut == 0 || first;               // not before the tile before has been read
    const auto load = [&](auto which, int h) {
      constexpr int W = decltype(which)::value;
      if (h < halves) half[W % AHEAD].template load<W % 2>(p, e, n0 / 16, tile0, direct, piece0 + h / 2, depths, groups, lane);
    };
    static_for<AHEAD>([&](auto u) { load(u, decltype(u)::value); });
    for (int h = 0; h < halves; h += TURN)
      static_for<TURN>([&](auto u) {
        constexpr int W = decltype(u)::value;
        if (h + W >= halves) return;
        half[W % AHEAD].template multiply<W % 2>(acc, depths - 4 * (piece0 + (h + W) / 2));
        load(Int<W + AHEAD>{}, h + W + AHEAD);
        if (W % 2 == 0) return;
        if (sums.last_piece()) {
          if (!may_write) __syncthreads();
          may_write = true;
          const int place = part == 0 ? 0 : 1 + sums.sum - (FEW_SUMS >> cut);
          const bool add = part == 0 && sums.sum > 0;         // (s0 is never without pieces)
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int t = 0; t < TG; ++t) {
              if constexpr (TOTAL) {
                if (part > 0) at_place(place, j, t) = acc[j][t];
                total[j][t] += acc[j][t];
              } else {
                if (add) acc[j][t] += at_place(place, j, t);
                at_place(place, j, t) = acc[j][t];
              }
              acc[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        sums.next();
      });
  } else if (cut > 0 && !first) {
    __syncthreads();
  }
  if (cut > 0) {
    if (TOTAL && TG > 1 && in && part == 0)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int t = 1; t < TG; ++t) at_place(0, j, t) = total[j][t];
    __syncthreads();
  }
  const int i = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < TG; ++t) {
    if (!in || part != (t & ((1 << cut) - 1))) continue;
    f32x4 sum[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) sum[j] = TOTAL && (t == 0 || cut == 0) ? total[j][t] : at_place(0, j, t);
    if (cut > 0) {
      const int own = FEW_SUMS >> cut;
      f32x4 other[FEW_SUMS][NB];
#pragma unroll
      for (int v = 1; v < FEW_SUMS; ++v)
#pragma unroll
        for (int j = 0; j < NB; ++j) other[v][j] = at_place(max(1 + v - own, 0), j, t);
#pragma unroll
      for (int v = 1; v < FEW_SUMS; ++v)
        if (v >= own && first_piece(v, SUMS_LOG2, groups) < first_piece(v + 1, SUMS_LOG2, groups))
#pragma unroll
          for (int j = 0; j < NB; ++j) sum[j] += other[v][j];
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
      uint8_t* const scales = p.Cs + ((size_t)(tile0 + t) * mx_groups(p.N) + depth / 4) * MX_SCALES;
      if (g == 0) scales[chunk * 64 + i * 4 + depth % 4] = (uint8_t)byte;
      if (DIRECT && n0 + FEW_COLS == p.N && p.N % 512 != 0) {      // the last columns' wavefront writes the zeros behind them
        if (g > chunk) *reinterpret_cast<u32x4*>(p.C + ((size_t)(tile0 + t) * mx_depths(p.N) + depth) * MX_TILE + lane * 16) = u32x4{0, 0, 0, 0};
        for (int q = g > chunk ? depth % 4 : depth % 4 + 1; q < 4; ++q) scales[g * 64 + i * 4 + q] = 0;
      }
    } else if (16 * t + i < rows) {
      bf16_t* out = p.O + ((size_t)p.off[e] + row_tile * TILE_ROWS + 16 * t + i) * p.N + n0 + 4 * g;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        *reinterpret_cast<u32x2*>(out + 16 * j) = u32x2{pack_bf16x2(sum[j][0], sum[j][1]), pack_bf16x2(sum[j][2], sum[j][3])};
    }
  }
}

// Tiles of the experts whose row count lies in (lo, hi], in ascending order of the experts; rows in tiles of TM.  An expert's tiles go through GROUP
// row tiles at a time, row tiles fastest, so that the tiles that an XCD multiplies at one time are a compact patch, whose operands its L2
// holds for all of them.
template <int TM, int GROUP>
struct SomeTiles {
  const int32_t* off;
  int e_cnt, lane, lo, hi;
  int n, incl, total, experts;
  __device__ __forceinline__ int count(int e) const {
    const int rows = e < e_cnt ? off[e + 1] - off[e] : 0;
    return rows > lo && rows <= hi ? (rows + TM - 1) / TM : 0;
  }
  __device__ __forceinline__ SomeTiles(const int32_t* __restrict__ off_, int e_cnt_, int lane_, int lo_, int hi_)
      : off(off_), e_cnt(e_cnt_), lane(lane_), lo(lo_), hi(hi_) {
    n = count(lane);
    incl = wave_scan(n);
    total = __builtin_amdgcn_readlane(incl, WAVE - 1);
    experts = __builtin_popcountll(__ballot(n > 0));
    for (int base = WAVE; base < e_cnt; base += WAVE) {
      const int more = count(base + lane);
      total += wave_sum(more);
      experts += __builtin_popcountll(__ballot(more > 0));
    }
  }
  // tile t < total n_cols
  __device__ __forceinline__ void at(int t, int n_cols, int& e, int& row_tile, int& col_tile) const {
    int rows = n, up_to = incl;
    for (int base = 0;; base += WAVE) {          // ends: t < total n_cols
      if (base > 0) up_to = wave_scan(rows = count(base + lane));
      const unsigned long long past = __ballot(up_to * n_cols > t);
      if (past) {
        const int who = __builtin_ctzll(past);
        e = base + who;
        rows = __builtin_amdgcn_readlane(rows, who);
        t -= (__builtin_amdgcn_readlane(up_to, who) - rows) * n_cols;
        const int group = t / (GROUP * n_cols), in_group = min(GROUP, rows - group * GROUP);
        t -= group * GROUP * n_cols;
        col_tile = t / in_group;
        row_tile = group * GROUP + t - col_tile * in_group;
        break;
      }
      t -= __builtin_amdgcn_readlane(up_to, WAVE - 1) * n_cols;
    }
    e = uniform(e);                              // (the compiler does not see that it is the same in all lanes)
    row_tile = uniform(row_tile);
    col_tile = uniform(col_tile);
  }
  // tile b of a walk that goes through every XCD's contiguous eighth; false: past its end
  __device__ __forceinline__ bool find(int n_cols, int b, int& e, int& row_tile, int& col_tile) const {
    const int share = (total * n_cols + 7) / 8, t = (b % 8) * share + b / 8;
    if (b / 8 >= share || t >= total * n_cols) return false;
    at(t, n_cols, e, row_tile, col_tile);
    return true;
  }
};

// ---- many rows per expert: 256 rows (the last of an expert: 256, 128 or 64) against 256 weight rows (UP: 128 of either matrix).  Eight
// wavefronts of 128 by 64 (64 by 64, 32 by 64) multiply in 32x32x64 instructions, two on each SIMD.  Operands go from memory to LDS
// directly, 128 of the contraction at a time, through a ring of four stages of which three are on their way.  Their layout in memory is
// the one that the instruction wants, so every load is 1 KB of consecutive bytes and every LDS read free of conflicts.  Workgroups are
// persistent, and the loads run ahead into the next tile while a finished one is written.
// Eight experts (4096 to 14336) of 1024 rows: 455 us up and 215 us down, a call 680 us, 4.2 PFLOP/s (a loop of these products on operands from LDS
// reaches 5.7, from registers 6.5), bound by the package's power: the matrix unit is busy half of the cycles at 1.9 GHz, and operands of zeros take
// 0.73 of the time.  Four stages are one turn of the loop, for the bytes of the scales' words to be chosen by the instruction (455 us; 465 with a
// byte read at every stage, 503 with shifted words).  A tile of up to 64 rows is a stream of weights, 0.7 us a stage.
constexpr int GEMM_GROUP = 4, GEMM_ROWS = 256, GEMM_COLS = 256, GEMM_THREADS = 512;
constexpr int STAGE = 32 * MX_TILE, STAGES = 4, SCALES = 32 * MX_SCALES;       // operand tiles of a stage: 16 of the rows, 16 of the weights
constexpr int PLACES = 3;                  // for scales (see Loads)
constexpr int GEMM_LDS = STAGES * STAGE + PLACES * SCALES;
constexpr int UP_LDS = GEMM_LDS > few_lds(4, 2) ? GEMM_LDS : few_lds(4, 2), DOWN_LDS = GEMM_LDS > few_lds(2, 2) ? GEMM_LDS : few_lds(2, 2), DIRECT_LDS = few_lds(4, 1);
static_assert(UP_LDS <= 160 * 1024 && DOWN_LDS <= 160 * 1024);
// (see Loads)  A contraction of up to 384 has fewer, and is a stream whatever the rows: 32 experts (384 to 384) of 2048 rows 162 us, of 416 to 416 77 us.
constexpr int LEAST_DEPTHS = 4;
__device__ __forceinline__ uint32_t next_place(uint32_t scales) { return scales == (PLACES - 1) * SCALES ? 0 : scales + SCALES; }
typedef float f32x16 __attribute__((ext_vector_type(16)));

// (scales: byte BYTE of the words)
template <int BYTE>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c, uint32_t sa, uint32_t sb) {
  const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, BYTE, (int)sa, BYTE, (int)sb);
}
// lanes 32..63 of a and lanes 0..31 of b change places
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
// until at most N of this wavefront's loads are on their way and its LDS reads are done, and until all wavefronts are there
template <int N>
__device__ __forceinline__ void wait_and_meet() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory"); }

typedef SomeTiles<GEMM_ROWS, GEMM_GROUP> GemmTiles;
template <int MODE, int NB>
struct Place {                             // of a tile
  int e = 0, row_tile = 0, col_tile = 0, rows = 0;      // rows: from its first row to the expert's end
  static constexpr int COLS = MODE == UP ? GEMM_COLS / 2 : GEMM_COLS / 2 * NB;
  __device__ __forceinline__ bool find(const XArgs& p, const GemmTiles& list, int b) {
    if (!list.find((p.N + COLS - 1) / COLS, b, e, row_tile, col_tile)) return false;
    rows = uniform(p.off[e + 1] - p.off[e]) - row_tile * GEMM_ROWS;
    return true;
  }
};

// The loads of a workgroup's tiles, stage after stage.  Of a stage wavefront w loads tiles 2 w and 2 w + 1 of the rows and of the weights (UP: 8 of
// W1, 8 of W3), four loads whatever the tile; those past the rows or columns repeat the last one (their results are not stored), and
// behind the last tile the same bytes are loaded again and again, so that the number of loads on their way is the same everywhere and the
// products' loop has no branch.  STREAM: the weights are read once.  The scales of 512 come with the first stage of the four.  Three of those have a place: the stages of a
// contraction's last scales may be fewer than the three that the loads are ahead, and with four stages to a contraction at least (LEAST_DEPTHS),
// two in succession belong to four stages or more, so that what is overwritten has been read.
template <int MODE, int NB, bool STREAM>
struct Loads {
  const XArgs& p;
  const GemmTiles& list;
  typedef Place<MODE, NB> AtPlace;
  AtPlace at;
  int b, t, depths, groups, lane, wave;
  bool more;
  uint32_t lds0, stage = 0, scales = 0;
  const uint8_t* a; const uint8_t* bw; const uint8_t* sc;
  uint32_t va[2], vb[NB], vsc;
  __device__ __forceinline__ Loads(const XArgs& p_, const GemmTiles& list_, uint32_t lds0_, int lane_, int wave_)
      : p(p_), list(list_), b(blockIdx.x), depths(mx_depths(p_.K)), groups(mx_groups(p_.K)), lane(lane_), wave(wave_), lds0(lds0_) {
    begin();
  }
  __device__ __forceinline__ void begin() {
    t = 0;
    more = at.find(p, list, b);
    const bool second = MODE == UP && wave >= 4;          // W3's
    const int first_b = second ? 2 * wave - 8 : NB * wave;
    // scales, four tiles' at a time: wavefronts 0 .. 3 the rows', 4 .. 7 the weights' (UP: 4 and 5 W1's)
    const bool of_weights = wave >= 4, of_second = MODE == UP && wave >= 6;
    const int first_s = 4 * (wave & (MODE == UP && of_weights ? 1 : 3));
    int last_a = 0, last_b = 0;
    if (more) {
      const int n0 = at.col_tile * AtPlace::COLS;
      const size_t tile0 = uniform(p.first[at.e]) + at.row_tile * (GEMM_ROWS / 16);
      last_a = (min(at.rows, GEMM_ROWS) + 15) / 16 - 1;
      last_b = min(AtPlace::COLS, p.N - n0) / 16 - 1;
      a = p.A + tile0 * depths * MX_TILE;
      bw = (second ? p.B1 : p.B0) + at.e * p.b_es + (size_t)(n0 / 16) * depths * MX_TILE;
      sc = of_weights ? (of_second ? p.Bs1 : p.Bs0) + at.e * p.bs_es + (size_t)(n0 / 16) * groups * MX_SCALES : p.As + tile0 * groups * MX_SCALES;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) va[j] = (uint32_t)(min(2 * wave + j, last_a) * depths * MX_TILE + lane * 16);
#pragma unroll
    for (int j = 0; j < NB; ++j) vb[j] = (uint32_t)(min(first_b + j, last_b) * depths * MX_TILE + lane * 16);
    vsc = (uint32_t)(min(first_s + lane / 16, of_weights ? last_b : last_a) * groups * MX_SCALES + lane % 16 * 16);
  }
  // before a stage's loads
  __device__ __forceinline__ void head() {
    if (t == depths) {
      b += gridDim.x;
      begin();
    }
    if (more && t % 4 == 0) {
      lds_load16((const bf16_t*)(sc + (size_t)(t / 4) * MX_SCALES), vsc, lds0 + STAGES * STAGE + scales + wave * 1024);
      scales = next_place(scales);
    }
  }
  // A stage's loads, one after the other: the caller spreads them over its products (issued in a row, a load keeps a wavefront for 80 cycles
  // while the others issue theirs).
  static constexpr int PARTS = NB + 2;
  template <int I>
  __device__ __forceinline__ void part() {
    const size_t from = (size_t)t * MX_TILE;
    if constexpr (I < NB) lds_load16<STREAM>((const bf16_t*)(bw + from), vb[I], lds0 + stage + (16 + NB * wave + I) * MX_TILE);
    else lds_load16((const bf16_t*)(a + from), va[I - NB], lds0 + stage + (2 * wave + I - NB) * MX_TILE);
    if (I == PARTS - 1) {
      stage = (stage + STAGE) % (STAGES * STAGE);
      t += more ? 1 : 0;
    }
  }
  __device__ __forceinline__ void issue() {
    head();
    static_for<PARTS>([&](auto i) { part<decltype(i)::value>(); });
  }
  // The next stage in order has arrived for all wavefronts, and all have done with the one that is to be loaded again.  The two stages behind it
  // are on their way.  (Scales, and at a tile's first stages the stores of the one before, are among what is on its way: they make the wait longer,
  // never shorter.)
  __device__ __forceinline__ void wait() { wait_and_meet<2 * PARTS>(); }
};

// A wavefront multiplies 32 * NA rows, half of the tile's, by 64 weight rows (UP: 32 of either matrix).  stage, scales: where this tile's first are.
template <int MODE, int NA, int NB, bool STREAM>
__device__ __forceinline__ void gemm_tile(const XArgs& p, Loads<MODE, NB, STREAM>& loads, const uint8_t* lds, uint32_t& stage, uint32_t& scales, const Place<MODE, NB>& at,
                                          int lane, int wave) {
  constexpr int HALF = NB / 2;             // 32-column operands; UP: HALF of either matrix
  const int depths = loads.depths, n0 = at.col_tile * Place<MODE, NB>::COLS;
  const int wr = wave & 1, wc = wave >> 1, h = lane >> 5;
  const auto b_tile = [&](int j) { return 16 + (MODE == UP ? 8 * j + 2 * wc : 2 * (NB * wc + j)); };
  const int in_tile = (lane >> 4 & 1) * MX_TILE + h * 256 + (lane & 15) * 16, in_scales = (lane >> 4 & 1) * MX_SCALES + h * 64 + (lane & 15) * 4;
  f32x16 acc[NA][NB];
#pragma unroll
  for (int i = 0; i < NA; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  u32x4 a[2][NA], b[2][NB];
  uint32_t as[2][NA], bs[2][NB];
  // operand I of step s (64 of the contraction) of the stage in place; with the first of four stages the scales of all of them
  const uint8_t* from;
  const uint8_t* scales_from;
  const auto read = [&](auto step, auto quarter, auto which) {
    // in the order in which the products take them: a weight operand, a row operand, the other weights, the other rows
    constexpr int s = decltype(step)::value, N = decltype(which)::value, I = N == 0 ? NA : N == 1 ? 0 : N <= NB ? NA + N - 1 : N - NB;
    if constexpr (I < NA) {
      a[s][I] = *reinterpret_cast<const u32x4*>(from + 512 * s + (2 * NA * wr + 2 * I) * MX_TILE);
      if constexpr (decltype(quarter)::value == 0) as[s][I] = *reinterpret_cast<const uint32_t*>(scales_from + 128 * s + (2 * NA * wr + 2 * I) * MX_SCALES);
    } else {
      b[s][I - NA] = *reinterpret_cast<const u32x4*>(from + 512 * s + b_tile(I - NA) * MX_TILE);
      if constexpr (decltype(quarter)::value == 0) bs[s][I - NA] = *reinterpret_cast<const uint32_t*>(scales_from + 128 * s + b_tile(I - NA) * MX_SCALES);
    }
  };
  // The products of a step, and between them the reads of the other one's operands and half of a stage's loads (of three the first, then two).
  constexpr int PRODUCTS = NA * NB, READS = NA + NB, READ_WITHIN = PRODUCTS < 4 ? PRODUCTS : 3 * PRODUCTS / 4, PARTS = Loads<MODE, NB, STREAM>::PARTS, FIRST = PARTS / 2;
  const auto multiply = [&](auto step, auto quarter) {               // quarter: of the stage whose operands are read
    constexpr int s = decltype(step)::value, Q = decltype(quarter)::value, MINE = s == 0 ? Q : (Q + 3) % 4, BEHIND = s == 0 ? FIRST : 0, LOADS = s == 0 ? PARTS - FIRST : FIRST;
    static_for<PRODUCTS>([&](auto m) {
      constexpr int M = decltype(m)::value, i = M / NB, j = M % NB;
      acc[i][j] = mfma32<MINE>(b[s][j], a[s][i], acc[i][j], bs[s][j], as[s][i]);
      constexpr int R0 = M * READS / READ_WITHIN, R = M < READ_WITHIN ? (M + 1) * READS / READ_WITHIN - R0 : 0;
      if constexpr (R > 0) static_for<R>([&](auto r) { read(Int<1 - s>{}, quarter, Int<R0 + decltype(r)::value>{}); });
      constexpr int L0 = M * LOADS / PRODUCTS, L = (M + 1) * LOADS / PRODUCTS - L0;
      if constexpr (L > 0) static_for<L>([&](auto l) { loads.template part<BEHIND + L0 + decltype(l)::value>(); });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // While one step's operands are multiplied the other's are on their way from LDS, across the barrier too, and the loads of the stage that
  // takes the place of the one before are issued.
  const auto begin = [&](int t) {
    loads.wait();
    loads.head();
    from = lds + stage + in_tile;
    scales_from = lds + STAGES * STAGE + scales + in_scales;
    stage = (stage + STAGE) % (STAGES * STAGE);
    if (t % 4 == 3 || t == depths - 1) scales = next_place(scales);
  };
  begin(0);
  static_for<READS>([&](auto r) { read(Int<0>{}, Int<0>{}, r); });
  static_for<FIRST>([&](auto l) { loads.template part<decltype(l)::value>(); });
  multiply(Int<0>{}, Int<0>{});
  int t = 1;
  const auto stage_of = [&](auto quarter) {
    begin(t);
    multiply(Int<1>{}, quarter);
    multiply(Int<0>{}, quarter);
    return ++t < depths;
  };
  if (t < depths)
    while (stage_of(Int<1>{}) && stage_of(Int<2>{}) && stage_of(Int<3>{}) && stage_of(Int<0>{})) {}
  const int behind = 8 * ((depths - 1) % 4);
#pragma unroll
  for (int i = 0; i < NA; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = mfma32<0>(b[1][j], a[1][i], acc[i][j], bs[1][j] >> behind, as[1][i] >> behind);
  // element 4 g + r of acc[i][j]: row lane % 32, column 8 g + 4 h + r of the 32
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    const int row = 32 * (NA * wr + i) + (lane & 31);
    if constexpr (MODE == UP) {
      const int tile = p.first[at.e] + at.row_tile * (GEMM_ROWS / 16) + row / 16;
#pragma unroll
      for (int j = 0; j < HALF; ++j) {
        float v[16];
        uint32_t top = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          v[r] = silu_f(acc[i][j][r]) * acc[i][j + HALF][r];
          top = max(top, __float_as_uint(v[r]) & 0x7FFFFFFFu);
        }
        uint32_t other = top;
        swap32(top, other);
        const uint32_t byte = mx_scale_byte(max(top, other));
        const float s = mx_scale_value(byte);
        uint32_t lo = byte == 255 ? 0u : mx_pack8(v, s), hi = byte == 255 ? 0u : mx_pack8(v + 8, s);
        swap32(lo, hi);                               // now bytes 8 h .. 8 h + 7 of the chunk, in halves of two lanes
        const u32x2 codes = {__builtin_amdgcn_perm(hi, lo, 0x05040100u), __builtin_amdgcn_perm(hi, lo, 0x07060302u)};
        const int col = n0 + 32 * (HALF * wc + j);
        if (row >= at.rows || col >= p.N) continue;
        const int depth = col / MX_DEPTH, chunk = col % MX_DEPTH / MX_CHUNK;
        *reinterpret_cast<u32x2*>(p.C + ((size_t)tile * mx_depths(p.N) + depth) * MX_TILE + chunk * 256 + row % 16 * 16 + 8 * h) = codes;
        if (h == 0) p.Cs[((size_t)tile * mx_groups(p.N) + depth / 4) * MX_SCALES + chunk * 64 + row % 16 * 4 + depth % 4] = (uint8_t)byte;
      }
    } else {
      bf16_t* const out = p.O + ((size_t)p.off[at.e] + at.row_tile * GEMM_ROWS + row) * p.N + n0 + 32 * NB * wc + 16 * h;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        uint32_t w[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) w[r] = pack_bf16x2(acc[i][j][2 * r], acc[i][j][2 * r + 1]);
#pragma unroll
        for (int r = 0; r < 4; ++r) swap32(w[r], w[r + 4]);         // columns 16 h .. 16 h + 15
        if (row >= at.rows || n0 + 32 * (NB * wc + j) >= p.N) continue;
        reinterpret_cast<u32x4*>(out + 32 * j)[0] = u32x4{w[0], w[1], w[4], w[5]};
        reinterpret_cast<u32x4*>(out + 32 * j)[1] = u32x4{w[2], w[3], w[6], w[7]};
      }
    }
  }
  // Where the lanes that stored meet the others: in a block of its own, for the compiler to see that what the walk keeps is the same in all
  // lanes (merged with the walk's own blocks, it kept LDS places and counters in vector registers).
  __builtin_amdgcn_wave_barrier();
}

// Workgroups walk the tiles of the experts with many rows, then those of the experts with few.
template <int MODE, bool STREAM, bool DIRECT = false>
__device__ __forceinline__ void few_tiles(const XArgs& p, const SomeTiles<DIRECT ? 16 : FEW_ROWS, 1>& list, f32x4* lds, int place, int idle, int rounds) {
  if (list.total == 0) return;
  // In how many wavefronts a tile's contraction is cut, and how many of the blocks of tiles the `idle` workgroups and the others, which have one
  // more of the large tiles behind them, take each.  Alone and few enough for every workgroup to have one: cut as far as they stay so.
  // Else the plan that ends first, in tenths of a large tile's stage: a block of tiles streams eight or four KB per wavefront in the place of
  // a stage's 16 KB, and begins and ends in what two stages take.
  const int cols = p.N / FEW_COLS, pieces = mx_groups(p.K);
  int split = FEW_WAVES, quota = 1, quota_others = 0;
  while (split > 1 && (split > pieces || list.total * ((cols * split + FEW_WAVES - 1) / FEW_WAVES) > (int)gridDim.x)) split /= 2;
  if (rounds > 0 || list.total * ((cols * split + FEW_WAVES - 1) / FEW_WAVES) > (int)gridDim.x) {
    const float stages = rounds > 0 ? 10.f * mx_depths(p.K) : 0.f, all = gridDim.x, others = all - idle;
    float best = __builtin_inff();
    for (int s = 1; s <= FEW_WAVES && s <= pieces; s *= 2) {
      const float n = (float)list.total * ((cols * s + FEW_WAVES - 1) / FEW_WAVES), cost = ((pieces + s - 1) / s) * (MODE == UP ? 48.f : 24.f) + 20.f;
      const float level = fmaxf(0.f, floorf((n * cost - idle * stages) / (all * cost)));          // of the others, in blocks of tiles
      for (float q = level; q < level + 2.f; q += 1.f) {
        const float qi = fmaxf(0.f, ceilf((n - others * q) / idle)), time = fmaxf(qi * cost, stages + q * cost);
        if (time < best) { best = time; split = s; quota_others = (int)q; }
      }
    }
    // (in integers: no tile may be left)
    const int rest = list.total * ((cols * split + FEW_WAVES - 1) / FEW_WAVES) - ((int)gridDim.x - idle) * quota_others;
    quota = rest > 0 ? (rest + idle - 1) / idle : 0;
  }
  const int cut = __builtin_ctz(uniform(split));
  quota = uniform(quota); quota_others = uniform(quota_others);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), per_block = FEW_WAVES >> cut, n_cols = (cols + per_block - 1) / per_block;
  const int n = list.total * n_cols, step = place < idle ? idle : gridDim.x - idle;
  int t = place < idle ? place : idle * quota + place - idle, e, row_tile, col_tile;
  bool first = true;
  for (int k = place < idle ? quota : quota_others; k > 0 && t < n; --k, t += step, first = false) {
    list.at(t, n_cols, e, row_tile, col_tile);
    const int rows = p.off[e + 1] - p.off[e] - row_tile * (DIRECT ? 16 : FEW_ROWS), n0 = (col_tile * per_block + (wave >> cut)) * FEW_COLS;
    if (DIRECT || rows <= 16) few_tile<MODE, 1, STREAM, DIRECT>(p, lds, cut, first, e, row_tile, n0, rows);
    else few_tile<MODE, 2, STREAM, false>(p, lds, cut, first, e, row_tile, n0, rows);
  }
}

template <int MODE, int NB, bool STREAM>
__device__ __forceinline__ void many_tiles(const XArgs& p, const GemmTiles& many, uint8_t* lds, int lane, int wave) {
  Place<MODE, NB> at;
  if (!at.find(p, many, blockIdx.x)) return;
  Loads<MODE, NB, STREAM> loads(p, many, lds_addr(lds), lane, wave);
  uint32_t stage = 0, scales = 0;
  loads.issue();
  loads.issue();
  loads.issue();
  for (int b = blockIdx.x;;) {
    if (at.rows > 128) gemm_tile<MODE, 4>(p, loads, lds, stage, scales, at, lane, wave);
    else if (at.rows > 64) gemm_tile<MODE, 2>(p, loads, lds, stage, scales, at, lane, wave);
    else gemm_tile<MODE, 1>(p, loads, lds, stage, scales, at, lane, wave);
    b += gridDim.x;
    if (!at.find(p, many, b)) break;
  }
  wait_and_meet<0>();                                 // LDS is the next tiles' own: what is still loaded has arrived, the last stage is read
}

template <int MODE>
__global__ __launch_bounds__(GEMM_THREADS, 1) void experts_mx4(XArgs p) {
  extern __shared__ uint8_t gemm_lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const GemmTiles many(p.off, p.e_cnt, lane, p.few_most, 0x7FFFFFFF);
  const SomeTiles<FEW_ROWS, 1> few(p.off, p.e_cnt, lane, 0, p.few_most);
  // Weights that are read once and that the Infinity Cache does not keep for the next call: 21 experts (7168 to 1536) of 64 rows read 5.5 TB/s with
  // the hint, 4.7 without, of 256 rows 3.7 and 3.4.  Eight experts of 1024 rows take 3 % longer with it, and what fits the cache 6 %.
  const bool once = many.experts + few.experts > p.cached && many.total < 2 * many.experts;
  // DOWN: half as many columns where that still leaves a workgroup to every tile, those of few rows with them (two halves are counted for a whole
  // one, also where the last columns have but one).  Eight experts (2880 to 2880) of
  // 200 rows: 16.5 us, 21.5 with whole ones.
  const bool half = MODE == DOWN && 2 * many.total * ((p.N + GEMM_COLS - 1) / GEMM_COLS) + few.total * ((p.N / FEW_COLS + FEW_WAVES - 1) / FEW_WAVES) <= (int)gridDim.x;
  if (half) many_tiles<MODE, MODE == DOWN ? 1 : 2, false>(p, many, gemm_lds, lane, wave);
  else if (once) many_tiles<MODE, 2, true>(p, many, gemm_lds, lane, wave);
  else many_tiles<MODE, 2, false>(p, many, gemm_lds, lane, wave);
  // the workgroups that had no tile in the others' last round come first: `idle` of them
  const int cols = half ? Place<MODE, 1>::COLS : Place<MODE, 2>::COLS;
  const int per_xcd = gridDim.x / 8, busy = ((many.total * ((p.N + cols - 1) / cols) + 7) / 8) % per_xcd;
  const int place = 8 * ((blockIdx.x / 8 + per_xcd - busy) % per_xcd) + blockIdx.x % 8, idle = 8 * (per_xcd - busy);
  if (few.total > p.cached) few_tiles<MODE, true>(p, few, reinterpret_cast<f32x4*>(gemm_lds), place, idle, many.total);
  else few_tiles<MODE, false>(p, few, reinterpret_cast<f32x4*>(gemm_lds), place, idle, many.total);
}

// UP of at most FEW_MOST rows in all, from bf16: a launch less.  The whole forward (4096 to 1536) of a row of one expert takes 13.3 us, 17.1 with
// expert_rows; of a row each of eight experts 22.6 and 26.4, of 32 experts 61 and 66.  An expert with 17 to 32 rows reads its weights twice: 20 rows
// of one alone (4096 to 14336) 37 us, 32 with expert_rows.
__global__ __launch_bounds__(GEMM_THREADS, 1) void up_direct(XArgs p) {
  extern __shared__ uint8_t gemm_lds[];
  const int lane = threadIdx.x & 63;
  if (blockIdx.x == 0 && threadIdx.x < WAVE) {
    int before = 0;
    for (int base = 0; base < p.e_cnt; base += WAVE) {
      const int i = base + lane, n = i < p.e_cnt ? (p.off[i + 1] - p.off[i] + 15) / 16 : 0, incl = wave_scan(n);
      if (i < p.e_cnt) p.first_out[i] = before + incl - n;
      before += __builtin_amdgcn_readlane(incl, WAVE - 1);
    }
  }
  const SomeTiles<16, 1> few(p.off, p.e_cnt, lane, 0, FEW_MOST);
  if (few.total > p.cached) few_tiles<UP, true, true>(p, few, reinterpret_cast<f32x4*>(gemm_lds), blockIdx.x, gridDim.x, 0);
  else few_tiles<UP, false, true>(p, few, reinterpret_cast<f32x4*>(gemm_lds), blockIdx.x, gridDim.x, 0);
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
  const long long tiles = tiles_bound(cap, e_cnt, 16);
  if (tiles * (d > f ? d : f) / FEW_COLS >= (1ll << 30)) return MOE_EUNSUPPORTED;       // tiles are counted in 32 bits
  const bool direct = cap <= FEW_MOST;
  if (!direct) {
    ProfScope prof(MOE_K_MX4_ROWS, s);
    const unsigned parts = (mx_groups(d) + ROWS_BLOCK / WAVE - 1) / (ROWS_BLOCK / WAVE);
    const int rc = in_launches(tiles, (int)parts * ROWS_BLOCK, [&](long long tile0, unsigned here) {
      hipLaunchKernelGGL(expert_rows, dim3(here, parts), dim3(ROWS_BLOCK), 0, s, (const bf16_t*)xp, offsets, e_cnt, d, f, base + at.xq, base + at.xs,
                         base + at.aq, base + at.as, first, (int)tile0);
    });
    if (rc != MOE_OK) return rc;
  }
  {
    static bool attr_set[64] = {};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return MOE_EHIP;
    if (!attr_set[dev]) {
      if (hipFuncSetAttribute(reinterpret_cast<const void*>(&experts_mx4<UP>), hipFuncAttributeMaxDynamicSharedMemorySize, UP_LDS) != hipSuccess ||
          hipFuncSetAttribute(reinterpret_cast<const void*>(&experts_mx4<DOWN>), hipFuncAttributeMaxDynamicSharedMemorySize, DOWN_LDS) != hipSuccess ||
          hipFuncSetAttribute(reinterpret_cast<const void*>(&up_direct), hipFuncAttributeMaxDynamicSharedMemorySize, DIRECT_LDS) != hipSuccess)
        return MOE_EHIP;
      attr_set[dev] = true;
    }
  }
  const dim3 walkers(8 * ((device_cu_count() + 7) / 8));       // (a walk stays in its XCD's eighth)
  XArgs p{};
  p.off = offsets; p.first = first; p.e_cnt = e_cnt;
  p.X = (const bf16_t*)xp; p.first_out = first;
  p.A = base + at.xq; p.As = base + at.xs;
  p.B0 = w1; p.Bs0 = s1; p.B1 = w3; p.Bs1 = s3;
  p.C = base + at.aq; p.Cs = base + at.as;
  p.N = f; p.K = d;
  p.few_most = mx_depths(p.K) < LEAST_DEPTHS ? 0x7FFFFFFF : FEW_MOST;
  p.cached = (int)((256ll << 20) * 32 / (51ll * d * f));
  p.b_es = (size_t)((f + 15) / 16) * mx_depths(d) * MX_TILE; p.bs_es = (size_t)((f + 15) / 16) * mx_groups(d) * MX_SCALES;
  {
    ProfScope prof(MOE_K_MX4_UP, s);
    if (direct) hipLaunchKernelGGL(up_direct, walkers, dim3(GEMM_THREADS), DIRECT_LDS, s, p);
    else hipLaunchKernelGGL(experts_mx4<UP>, walkers, dim3(GEMM_THREADS), UP_LDS, s, p);
    HIP_CHECK_LAUNCH();
  }
  p.A = p.C; p.As = p.Cs;
  p.B0 = w2; p.Bs0 = s2; p.B1 = nullptr; p.Bs1 = nullptr;
  p.O = (bf16_t*)o;
  p.N = d; p.K = f;
  p.few_most = mx_depths(p.K) < LEAST_DEPTHS ? 0x7FFFFFFF : FEW_MOST;
  p.b_es = (size_t)((d + 15) / 16) * mx_depths(f) * MX_TILE; p.bs_es = (size_t)((d + 15) / 16) * mx_groups(f) * MX_SCALES;
  {
    ProfScope prof(MOE_K_MX4_DOWN, s);
    hipLaunchKernelGGL(experts_mx4<DOWN>, walkers, dim3(GEMM_THREADS), DOWN_LDS, s, p);
    HIP_CHECK_LAUNCH();
  }
  return MOE_OK;
}
