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

template <int MODE>
__global__ __launch_bounds__(FEW_WAVES * WAVE) void few_rows_mx4(XArgs p) {
  __shared__ f32x4 lds[FEW_WAVES * (MODE == UP ? 4 : 2) * WAVE];
  const RaggedTiles<FEW_ROWS> list(p.off, p.e_cnt, threadIdx.x & 63);
  int e, row_tile, col_tile;
  if (!list.tile(p.N / FEW_COLS, blockIdx.x, e, row_tile, col_tile)) return;
  const int rows = p.off[e + 1] - p.off[e] - row_tile * FEW_ROWS;
  if (rows <= 16) few_tile<MODE, 1>(p, lds, e, row_tile, col_tile * FEW_COLS, rows);
  else few_tile<MODE, 2>(p, lds, e, row_tile, col_tile * FEW_COLS, rows);
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
  XArgs p{};
  p.off = offsets; p.first = first; p.e_cnt = e_cnt;
  p.A = base + at.xq; p.As = base + at.xs;
  p.B0 = w1; p.Bs0 = s1; p.B1 = w3; p.Bs1 = s3;
  p.C = base + at.aq; p.Cs = base + at.as;
  p.N = f; p.K = d;
  p.b_es = (size_t)((f + 15) / 16) * mx_depths(d) * MX_TILE; p.bs_es = (size_t)((f + 15) / 16) * mx_groups(d) * MX_SCALES;
  {
    ProfScope prof(MOE_K_MX4_UP, s);
    hipLaunchKernelGGL(few_rows_mx4<UP>, dim3((unsigned)up), dim3(WAVE * min(FEW_WAVES, mx_groups(d))), 0, s, p);
    HIP_CHECK_LAUNCH();
  }
  p.A = p.C; p.As = p.Cs;
  p.B0 = w2; p.Bs0 = s2; p.B1 = nullptr; p.Bs1 = nullptr;
  p.O = (bf16_t*)o;
  p.N = d; p.K = f;
  p.b_es = (size_t)((d + 15) / 16) * mx_depths(f) * MX_TILE; p.bs_es = (size_t)((d + 15) / 16) * mx_groups(f) * MX_SCALES;
  {
    ProfScope prof(MOE_K_MX4_DOWN, s);
    hipLaunchKernelGGL(few_rows_mx4<DOWN>, dim3((unsigned)down), dim3(WAVE * min(FEW_WAVES, mx_groups(f))), 0, s, p);
    HIP_CHECK_LAUNCH();
  }
  return MOE_OK;
}
