// Microscaled 4-bit numbers in memory, and the conversions of one 32-element chunk.
//
// A number is e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives, codes in that order, sign in bit 3) times a power of two that 32 elements
// along the contraction share, kept as its exponent plus 127 in a byte.  n rows of K elements are stored in the order in which the matrix
// instruction takes them, so that a wavefront's operand of 16 rows by 128 elements is 1 KB of consecutive memory, 16 bytes per lane:
//   data    [n/16][K/128][4 chunks][16 rows][16 bytes]              a chunk's 32 elements, the even ones in the low half of their byte
//   scales  [n/16][K/512][4 chunks][16 rows][4 pieces of 128]       a lane's scales of four operands are four bytes of one word
// Rows and elements past n and K are zeros, data and scales.
#pragma once
#include "common.h"

namespace {

typedef unsigned int mx_u32x4 __attribute__((ext_vector_type(4)));

constexpr int MX_ROWS = 16, MX_DEPTH = 128, MX_CHUNK = 32;
constexpr int MX_TILE = 1024, MX_SCALES = 256;         // bytes: data of 16 x 128, scales of 16 x 512
__host__ __device__ inline int mx_depths(int K) { return (K + 127) / 128; }
__host__ __device__ inline int mx_groups(int K) { return (K + 511) / 512; }

// Scale byte of a chunk from the bits of its largest magnitude as fp32: the power of two below it goes to 4, the one in e2m1's largest binade
// (what lies in (6, 8) then saturates at 6); not below 2^-127.  Infinities and NaN give 255, a NaN scale.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top_bits) {
  const int e = (int)(top_bits >> 23);
  return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}

// Eight floats to eight codes, round to nearest even.
// The conversion divides by the scale given as a float of that exponent; 2^-127 is one of fp32's denormal numbers.
__device__ __forceinline__ float mx_scale_value(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }
__device__ __forceinline__ uint32_t mx_pack8(const float* v, float scale) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
}
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t mx_pack8(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float scale) {      // pairs of bf16
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, a), scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, b), scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, c), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, d), scale, 3);
}
__device__ __forceinline__ uint32_t mx_top(uint32_t a, uint32_t b) {          // larger magnitudes of two pairs of bf16, without signs
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a & 0x7FFF7FFFu), __builtin_bit_cast(u16x2, b & 0x7FFF7FFFu)));
}
__device__ __forceinline__ uint32_t mx_top_bits(uint32_t pair) { return max(pair << 16, pair & 0xFFFF0000u); }      // of a pair, as fp32

// 32 consecutive elements: 16 words of bf16 pairs, or 32 floats
__device__ __forceinline__ mx_u32x4 mx_chunk(const uint32_t (&w)[16], uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = mx_top(top, w[i]);
  byte = mx_scale_byte(mx_top_bits(top));
  const float s = mx_scale_value(byte);
  mx_u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = byte == 255 ? 0u : mx_pack8(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3], s);
  return r;
}
__device__ __forceinline__ mx_u32x4 mx_chunk(const float (&v)[32], uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  byte = mx_scale_byte(top);
  const float s = mx_scale_value(byte);
  mx_u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = byte == 255 ? 0u : mx_pack8(v + 8 * i, s);
  return r;
}

// Eight consecutive elements of a lane (a chunk is four lanes side by side) as loaded, and their codes.
template <typename T> struct Mx8;
template <> struct Mx8<bf16_t> {
  mx_u32x4 v;
  __device__ __forceinline__ void load(const bf16_t* p) { v = __builtin_nontemporal_load(reinterpret_cast<const mx_u32x4*>(p)); }
  __device__ __forceinline__ void zero() { v = mx_u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ uint32_t top() const { return mx_top_bits(mx_top(mx_top(v[0], v[1]), mx_top(v[2], v[3]))); }
  __device__ __forceinline__ uint32_t codes(float s) const { return mx_pack8(v[0], v[1], v[2], v[3], s); }
};
template <> struct Mx8<float> {
  mx_u32x4 v[2];
  __device__ __forceinline__ void load(const float* p) {
    v[0] = __builtin_nontemporal_load(reinterpret_cast<const mx_u32x4*>(p));
    v[1] = __builtin_nontemporal_load(reinterpret_cast<const mx_u32x4*>(p) + 1);
  }
  __device__ __forceinline__ void zero() { v[0] = v[1] = mx_u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, v[i / 4][i % 4] & 0x7FFFFFFFu);
    return t;
  }
  __device__ __forceinline__ uint32_t codes(float s) const {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[i / 4][i % 4]);
    return mx_pack8(f, s);
  }
};
// largest of four lanes side by side
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));      // quad_perm 1 0 3 2
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));   // quad_perm 2 3 0 1
}

// A wavefront's tiles of 16 rows by 512 elements from rows that are contiguous: 16 lanes load 128 elements of a row, so that a load takes 256
// consecutive bytes (fp32: 512) of each of four rows, and a chunk's largest magnitude is found across four lanes.
// src: element 0 of the first row; rows, K: what of it there is (the rest is zeros); tile, group: where it goes.
template <typename T>
__device__ __forceinline__ void mx_rows_512(const T* src, int rows, int K, size_t tile, int group, int lane, uint8_t* __restrict__ q, uint8_t* __restrict__ scales) {
  const int groups = mx_groups(K), depths = mx_depths(K), r0 = lane >> 4, c = lane & 15;
  Mx8<T> x[4][4];
#pragma unroll
  for (int p = 0; p < 4; ++p)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = 512 * group + MX_DEPTH * p + 8 * c, row = 4 * j + r0;
      if (row < rows && k < K) x[p][j].load(src + (size_t)row * K + k);
      else x[p][j].zero();
    }
  uint32_t word[4] = {0, 0, 0, 0};
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int depth = 4 * group + p;
    if (depth >= depths) break;
    uint8_t* const out = q + (tile * depths + depth) * MX_TILE + (c >> 2) * 256 + (c & 3) * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t byte = mx_scale_byte(quad_max(x[p][j].top()));
      word[j] |= byte << (8 * p);
      *reinterpret_cast<uint32_t*>(out + (4 * j + r0) * 16) = byte == 255 ? 0u : x[p][j].codes(mx_scale_value(byte));
    }
  }
  if ((c & 3) == 0)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint32_t*>(scales + (tile * groups + group) * MX_SCALES + (c >> 2) * 64 + (4 * j + r0) * 4) = word[j];
}

}  // namespace
