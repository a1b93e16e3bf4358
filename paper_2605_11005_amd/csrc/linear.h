// Launch functions of the linear layer, grouped by expert or dense: linear.hip, with its products in linear_few.hip, linear_tiles.hip,
// expert_bf16.hip (the large ones) and expert_f32.hip.
#pragma once
#include "kernels.h"

struct LinearArgs {
  const void *x, *w, *bias, *residual;
  void *z, *y;
  int dtype, rows, K, N, e_cnt, act;
  const int32_t* offsets;                 // NULL: one matrix, all rows
};
// db[e] (+)= the sums of expert e's row tiles of LINEAR_SUM_ROWS rows: lines off[e] / LINEAR_SUM_ROWS + e and on of sums (bias_grad.h), or of its rows
// themselves, dy act'(z); db NULL: none
constexpr int LINEAR_SUM_ROWS = 64;
struct BiasGrad {
  const int32_t* off;                     // NULL: one expert, all rows
  int rows, N, accumulate;
  const float* sums;
  const void *dy, *z;                     // dy NULL: sums
  int act;
  void* db;
};
size_t linear_fwd_ws_bytes(int dtype, int rows, int K, int N, int e_cnt);
size_t linear_bwd_ws_bytes(int dtype, int rows, int K, int N, int e_cnt);
int launch_linear_fwd(const LinearArgs& l, void* ws, hipStream_t s);
int launch_linear_bwd(const LinearArgs& l, const void* dy, void* dx, int dx_accumulate, void* dw, void* db, int accumulate, void* ws, hipStream_t s);
size_t linear_few_ws_bytes(int rows, int N);
int launch_linear_few(const LinearArgs& l, void* ws, hipStream_t s);
int launch_linear_tiles_fwd(const LinearArgs& l, void* ws, hipStream_t s);
int launch_linear_tiles_bwd(const LinearArgs& l, const void* dz, void* dx, int dx_accumulate, void* dw, int accumulate, const BiasGrad& db, void* ws_dx, void* ws_dw,
                            hipStream_t s);
float linear_tiles_fwd_time(const LinearArgs& l);                    // in us, by the model that cuts their contractions
float linear_tiles_bwd_time(const LinearArgs& l, bool dx, bool dw);
size_t linear_parts_bytes(long long rows, int columns);
int launch_linear_fwd_large(const LinearArgs& l, int32_t* sched, hipStream_t s);
size_t linear_split_bytes(int K, int N);
int launch_linear_bwd_large(const LinearArgs& l, const void* dz, void* dx, int dx_accumulate, void* dw, int accumulate, int32_t* sched, void* ws, hipStream_t s);
size_t linear_f32_parts_bytes(long long rows, int columns);
int launch_linear_fwd_f32(const LinearArgs& l, void* ws, hipStream_t s);
int launch_linear_bwd_f32(const LinearArgs& l, const void* dz, void* dx, int dx_accumulate, void* dw, int accumulate, const BiasGrad& db, void* ws_dx, void* ws_dw,
                          hipStream_t s);
