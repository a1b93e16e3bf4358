// Quantisation to microscaled 4 bits and back (layout and rounding: mx4.h).  HBM bound: every element is read once and every byte
// written once.
#include "mx4.h"
#include "kernels.h"

namespace {

typedef unsigned int mx_u32x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));
constexpr int QUANT_BLOCK = 256;

// Rows whose elements are contiguous (tokens): a wavefront per 16 rows by 512 elements, 64 KB of loads on their way per CU and more.  2047 rows of
// 2880 bf16: 5 us, a launch; 16249 rows of 7168 50 us, 5.9 TB/s, fp32 104, 5.1.
template <typename T>
__global__ __launch_bounds__(QUANT_BLOCK) void mx4_rows(const T* __restrict__ x, int n, int K, long long first, long long jobs, uint8_t* __restrict__ q,
                                                         uint8_t* __restrict__ scales) {
  const long long job = (first + blockIdx.x) * (QUANT_BLOCK / WAVE) + (threadIdx.x >> 6);
  if (job >= jobs) return;
  const int groups = mx_groups(K), tiles = (n + 15) / 16, group = (int)(job % groups);
  const long long rest = job / groups, batch = rest / tiles;
  const int row0 = 16 * (int)(rest - batch * tiles);
  mx_rows_512(x + ((size_t)batch * n + row0) * K, n - row0, K, (size_t)rest, group, threadIdx.x & 63, q, scales);
}

// Matrices [K][n] whose contraction index is not the contiguous one (weights).  A lane takes four columns of 32 rows; the four
// wavefronts of a block take the same chunk of four consecutive operands, whose scales meet in LDS as the bytes of a word.  16 matrices of
// 4096 by 1536, bf16: 46 us, 5.5 TB/s (62 us without the hint that no element is read again), fp32 78 us, 5.9 TB/s.
template <typename T>
__global__ __launch_bounds__(QUANT_BLOCK) void mx4_columns(const T* __restrict__ x, int n, int K, int first, int col_blocks, uint8_t* __restrict__ q,
                                                            uint8_t* __restrict__ scales) {
  __shared__ uint8_t bytes[QUANT_BLOCK * 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int groups = mx_groups(K), depths = mx_depths(K), tiles = (n + 15) / 16;
  int b = first + blockIdx.x;
  const int col_block = b % col_blocks; b /= col_blocks;
  const int chunk = b % 4; b /= 4;
  const int group = b % groups, batch = b / groups;
  const int col = col_block * QUANT_BLOCK + 4 * lane, depth = 4 * group + wave, k = MX_DEPTH * depth + MX_CHUNK * chunk;
  uint32_t byte[4] = {0, 0, 0, 0};
  mx_u32x4 codes[4] = {};
  if (col < n && k < K) {
    const T* src = x + ((size_t)batch * K + k) * n + col;
    if constexpr (sizeof(T) == 2) {
      mx_u32x2 v[MX_CHUNK];
#pragma unroll
      for (int i = 0; i < MX_CHUNK; ++i) v[i] = __builtin_nontemporal_load(reinterpret_cast<const mx_u32x2*>(src + (size_t)i * n));
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
          w[i] = __builtin_amdgcn_perm(c < 2 ? v[2 * i + 1].x : v[2 * i + 1].y, c < 2 ? v[2 * i].x : v[2 * i].y, c & 1 ? 0x07060302u : 0x05040100u);
        codes[c] = mx_chunk(w, byte[c]);
      }
    } else {
      mx_f32x4 v[MX_CHUNK];
#pragma unroll
      for (int i = 0; i < MX_CHUNK; ++i) v[i] = __builtin_nontemporal_load(reinterpret_cast<const mx_f32x4*>(src + (size_t)i * n));
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float w[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = c == 0 ? v[i].x : c == 1 ? v[i].y : c == 2 ? v[i].z : v[i].w;
        codes[c] = mx_chunk(w, byte[c]);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) bytes[(4 * lane + c) * 4 + wave] = (uint8_t)byte[c];
  if (depth < depths && col < 16 * tiles) {
    uint8_t* dst = q + (((size_t)batch * tiles + (col >> 4)) * depths + depth) * MX_TILE + chunk * 256 + (col & 15) * 16;
#pragma unroll
    for (int c = 0; c < 4; ++c) reinterpret_cast<mx_u32x4*>(dst)[c] = codes[c];
  }
  __syncthreads();
  const int own = col_block * QUANT_BLOCK + threadIdx.x;
  if (own < 16 * tiles)
    *reinterpret_cast<uint32_t*>(scales + (((size_t)batch * tiles + (own >> 4)) * groups + group) * MX_SCALES + chunk * 64 + (own & 15) * 4) =
        *reinterpret_cast<const uint32_t*>(bytes + 4 * threadIdx.x);
}

// Back to values [n][K]: exact in either type (an e2m1 number has two bits of mantissa).  A block takes 16 rows by 512 elements, a lane
// 16 bytes of every store, so that 16 lanes write 256 bytes of a row.  16 matrices of 4096 by 1536 to bf16: 48 us, 5.3 TB/s, right behind
// their quantisation, when the Infinity Cache holds the codes, 38; to fp32 97 us, 4.7 TB/s.
template <typename T>
__global__ __launch_bounds__(QUANT_BLOCK) void mx4_values(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scales, int n, int K, unsigned first,
                                                           T* __restrict__ out) {
  constexpr int N = 16 / sizeof(T), STORES = MX_DEPTH / (16 * N);             // elements of a lane in a store, stores of an operand's row
  const int groups = mx_groups(K), depths = mx_depths(K), tiles = (n + 15) / 16;
  const unsigned at_block = first + blockIdx.x;
  const int group = at_block % groups, rest = at_block / groups, batch = rest / tiles;
  const int i = threadIdx.x >> 4, c = threadIdx.x & 15;                       // row, N elements of each store's
  const int row = 16 * (rest - batch * tiles) + i;
  if (row >= n) return;
  T* dst = out + ((size_t)batch * n + row) * K;
#pragma unroll
  for (int st = 0; st < STORES; ++st) {
    const int at = 16 * N * st + N * c, chunk = at / MX_CHUNK;                // of the 128
    const uint32_t word = *reinterpret_cast<const uint32_t*>(scales + ((size_t)rest * groups + group) * MX_SCALES + chunk * 64 + i * 4);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int depth = 4 * group + p, k = MX_DEPTH * depth + at;
      if (k >= K) break;
      const uint8_t* codes = q + ((size_t)rest * depths + depth) * MX_TILE + chunk * 256 + i * 16 + at % MX_CHUNK / 2;
      const uint32_t v = N == 8 ? *reinterpret_cast<const uint32_t*>(codes) : *reinterpret_cast<const uint16_t*>(codes);
      const uint32_t byte = (word >> (8 * p)) & 255u;
      const float s = byte == 255 ? __uint_as_float(0x7FC00000u) : mx_scale_value(byte);
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      // codes as multiples of 1/2, times the scale: both steps are exact
      const f32x2 e0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.f, 0), e1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.f, 1);
      if constexpr (N == 8) {
        const f32x2 e2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.f, 2), e3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.f, 3);
        *reinterpret_cast<mx_u32x4*>(dst + k) = mx_u32x4{pack_bf16x2(e0.x * s, e0.y * s), pack_bf16x2(e1.x * s, e1.y * s),
                                                         pack_bf16x2(e2.x * s, e2.y * s), pack_bf16x2(e3.x * s, e3.y * s)};
      } else {
        *reinterpret_cast<mx_f32x4*>(dst + k) = mx_f32x4{e0.x * s, e0.y * s, e1.x * s, e1.y * s};
      }
    }
  }
}

}  // namespace

int launch_mx4_quantize(const void* x, int dtype, int batch, int n, int K, int along_rows, uint8_t* q, uint8_t* scales, hipStream_t s) {
  if (batch == 0 || n == 0 || K == 0) return MOE_OK;
  ProfScope prof(MOE_K_MX4_QUANTIZE, s);
  if (along_rows) {
    const int col_blocks = (n + QUANT_BLOCK - 1) / QUANT_BLOCK;
    const long long blocks = (long long)batch * mx_groups(K) * 4 * col_blocks;
    if (blocks >= (1ll << 31)) return MOE_EUNSUPPORTED;
    return in_launches(blocks, QUANT_BLOCK, [&](long long first, unsigned here) {
      if (dtype == MOE_BF16)
        hipLaunchKernelGGL(mx4_columns<bf16_t>, dim3(here), dim3(QUANT_BLOCK), 0, s, (const bf16_t*)x, n, K, (int)first, col_blocks, q, scales);
      else
        hipLaunchKernelGGL(mx4_columns<float>, dim3(here), dim3(QUANT_BLOCK), 0, s, (const float*)x, n, K, (int)first, col_blocks, q, scales);
    });
  }
  const long long jobs = (long long)batch * ((n + 15) / 16) * mx_groups(K);
  return in_launches((jobs + QUANT_BLOCK / WAVE - 1) / (QUANT_BLOCK / WAVE), QUANT_BLOCK, [&](long long first, unsigned here) {
    if (dtype == MOE_BF16)
      hipLaunchKernelGGL(mx4_rows<bf16_t>, dim3(here), dim3(QUANT_BLOCK), 0, s, (const bf16_t*)x, n, K, first, jobs, q, scales);
    else
      hipLaunchKernelGGL(mx4_rows<float>, dim3(here), dim3(QUANT_BLOCK), 0, s, (const float*)x, n, K, first, jobs, q, scales);
  });
}

int launch_mx4_dequantize(const uint8_t* q, const uint8_t* scales, int batch, int n, int K, void* out, int dtype, hipStream_t s) {
  if (batch == 0 || n == 0 || K == 0) return MOE_OK;
  ProfScope prof(MOE_K_MX4_DEQUANTIZE, s);
  // (fewer than 2^31 workgroups: the entry point refuses more tiles)
  return in_launches((long long)batch * ((n + 15) / 16) * mx_groups(K), QUANT_BLOCK, [&](long long first, unsigned here) {
    if (dtype == MOE_BF16)
      hipLaunchKernelGGL(mx4_values<bf16_t>, dim3(here), dim3(QUANT_BLOCK), 0, s, q, scales, n, K, (unsigned)first, (bf16_t*)out);
    else
      hipLaunchKernelGGL(mx4_values<float>, dim3(here), dim3(QUANT_BLOCK), 0, s, q, scales, n, K, (unsigned)first, (float*)out);
  });
}
