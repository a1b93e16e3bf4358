// Operands of a 128x128 tile whose k-tiles are 64 deep, 16 KB each: from memory straight into LDS by whole cache lines, and from there into
// the registers of v_mfma_f32_32x32x16_bf16.
//   K-contiguous operand   [128 rows][8 chunks of 8 k]       chunk' = chunk ^ ((row>>1)&7)
//   transposed operand     2 x [64 k][8 chunks of 8 n]       chunk' = chunk ^ (4*((k>>1)&1))
#pragma once
#include "common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int QT = 128, QK = 64;
constexpr int QOPER_BYTES = QT * QK * 2;

// Bytes that a load of the chunk of 8 k at k goes back by so as not to read past the contraction's K
__device__ __forceinline__ uint32_t past_end(int k, int K) { return 2u * (uint32_t)max(0, k - (K - 8)); }

__device__ __forceinline__ bf16x8 lds_frag_kc(const char* p) { return *reinterpret_cast<const bf16x8*>(p); }
struct QuarterKc {         // load j of a wavefront: rows 8*(4w+j) + lane/8, whole 128-byte lines
  const bf16_t* base;
  uint32_t voff[4];
  __device__ __forceinline__ void setup(const bf16_t* base_, long ld, int rows_valid, int wave, int lane) {
    base = base_;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int rl = 8 * (4 * wave + j) + (lane >> 3);
      const int c = (lane & 7) ^ ((rl >> 1) & 7);
      voff[j] = (uint32_t)(min(rl, rows_valid - 1) * ld * 2 + c * 16);
    }
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void issue1(int j, uint32_t oper_lds, int wave, long kofs, uint32_t back = 0) const {
    lds_load16<STREAM>(base + kofs, voff[j] - back, oper_lds + (4 * wave + j) * 1024);
  }
  static __device__ __forceinline__ int chunk(int j, int lane) { return (lane & 7) ^ (4 * (j & 1) + (lane >> 4)); }
};
struct QuarterTr {         // sub-tile wave/2, load j: k rows 8*(4*(w%2)+j) + lane/8, 64 columns each
  const bf16_t* src;
  long ld;
  uint32_t coff;
  __device__ __forceinline__ void setup(const bf16_t* b0, const bf16_t* b1, bool dual, long ld_, int n0, int n_lim, int wave, int lane) {
    ld = ld_;
    const int sub = wave >> 1, c = (lane & 7) ^ (4 * ((lane >> 4) & 1));
    src = (dual && sub) ? b1 : b0;
    coff = (uint32_t)(2 * min(n0 + (dual ? 0 : sub * 64) + c * 8, n_lim - 8));
  }
  template <bool CLAMP, bool STREAM = false>    // source rows above k_last_rel are clamped (the caller zeroes the matching A fragments)
  __device__ __forceinline__ void issue1(int j, uint32_t oper_lds, int wave, int lane, long k0, int k_last_rel) const {
    int kr = 8 * (4 * (wave & 1) + j) + (lane >> 3);
    if (CLAMP && kr > k_last_rel) kr = k_last_rel;
    lds_load16<STREAM>(src + k0 * ld, (uint32_t)(kr * ld * 2) + coff, oper_lds + (4 * wave + j) * 1024);
  }
};
// transposed sub-tile: byte offset of the first transposing read of 32 columns at nl (0 or 32), k-step 0; add s*2048 + t*512
__device__ __forceinline__ int quarter_tr_off(int sub, int nl, int lane) {
  const int i = lane & 15, g = lane >> 4;
  const int k = 8 * (g >> 1) + (i >> 2);
  const int n = nl + 16 * (g & 1) + 4 * (i & 3);
  return sub * 8192 + k * 128 + (((n >> 3) ^ (4 * ((k >> 1) & 1))) << 4) + ((n & 4) << 1);
}
__device__ __forceinline__ bf16x8 quarter_frag_tr(const char* p) {
  s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p));
  s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 512));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

}  // namespace
