// Operands of v_mfma_f32_16x16x32_bf16 from matrices whose contraction runs along the rows, through registers alone: a lane loads C columns of
// each of eight rows and turns the block, so that its column j is an operand of eight k.
#pragma once
#include "common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Loads go through a buffer descriptor: a wave-uniform base and a 32-bit byte offset per lane (64-bit addresses per lane limit a CU's address path,
// see lds_load16 in common.h).  A descriptor of length zero makes a load return zeros without touching memory.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const bf16_t* base, bool in) {
  uint64_t b = (uint64_t)base;
  int bytes = in ? 0x7FFFFFFF : 0;
  asm("" : "+s"(b), "+s"(bytes));         // both are wave-uniform: keep them in scalar registers
  return __builtin_amdgcn_make_buffer_rsrc((void*)b, 0, bytes, 0x00027000);
}

// A wavefront's piece of a matrix whose columns are contiguous: a lane holds C columns of each of eight rows.
template <int C>
struct ColumnPiece {
  unsigned int w[8][C / 2];
  template <bool STREAM>
  __device__ __forceinline__ void load(const bf16_t* base, bool in, int row, int voff) {
    constexpr int NT = STREAM ? 2 : 0;
    const __amdgpu_buffer_rsrc_t d = descriptor(base, in);
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      if constexpr (C == 8) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(d, voff, r * row, NT);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[r][q] = v[q];
      } else {
        const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(d, voff, r * row, NT);
        w[r][0] = v[0];
        w[r][1] = v[1];
      }
    }
  }
  // of rows first, first + 1, .. of `left` (1 or more): zeros past the last one
  __device__ __forceinline__ void load_end(const bf16_t* base, int row, int first, int left, int voff) {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const __amdgpu_buffer_rsrc_t d = descriptor(base, true);
      const int at = voff + min(first + r, left - 1) * row;
      const bool in = first + r < left;
      if constexpr (C == 8) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(d, at, 0, 0);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[r][q] = in ? v[q] : 0;
      } else {
        const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(d, at, 0, 0);
        w[r][0] = in ? v[0] : 0;
        w[r][1] = in ? v[1] : 0;
      }
    }
  }
  __device__ __forceinline__ bf16x8 operand(int j) const {      // column j of the block, its eight rows
    u32x4 f;
#pragma unroll
    for (int q = 0; q < 4; ++q) f[q] = __builtin_amdgcn_perm(w[2 * q + 1][j >> 1], w[2 * q][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
    return __builtin_bit_cast(bf16x8, f);
  }
};

}  // namespace
