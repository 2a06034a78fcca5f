// The gated block's products on tiles of 64 x 64 (small_tile.hip), bf16; widths are multiples of 64:
//   z2z_launch_small_gated    F = act(X W[:d_ff]^T) * (X W[d_ff:]^T), [R, d_ff]; kept: what the backward pass is given, or nothing
//   z2z_launch_small_slopes   dF = dY W, W [K, d_ff], as dG | dU [R, 2 d_ff]
//   z2z_launch_small_linear   out [R, N] = A [R, K] W^T + residual, W [N, K]; f32: residual and out are fp32
//   z2z_launch_small_parts    A W^T as fp32 parts [*ksplit][R][N], which the caller adds up before the next dense layer is launched; or nothing (0) where K is not shared out
//   z2z_launch_small_input    out [R, N] = A [R, K] W, W [K, N]
// rows_dev: nullptr, or how many of the R rows exist.  weight: nullptr, or a weight gradient over the same rows that goes along in the launch, out [M, N] =
// A [R, M]^T W [R, N] + residual.
#pragma once

#include "z2z_internal.h"

struct z2z_small_weight {
  const void *A, *W, *residual;
  void* out;
  int M, N;
};

int z2z_launch_small_gated(const void* X, const void* W, int act, void* F, const z2z_ffn_kept& kept, int R, const int32_t* rows_dev, int d_ff, int K, hipStream_t s);
int z2z_launch_small_slopes(z2z_ctx* c, const void* dY, const void* W, const z2z_ffn_kept& kept, void* slopes, int R, const int32_t* rows_dev, int d_ff, int K,
                            const z2z_small_weight* weight, hipStream_t s);
int z2z_launch_small_linear(z2z_ctx* c, const void* A, const void* W, const void* residual, void* out, bool f32, int R, const int32_t* rows_dev, int N, int K,
                            hipStream_t s);
int z2z_launch_small_parts(z2z_ctx* c, const void* A, const void* W, int R, const int32_t* rows_dev, int N, int K, const float** partial, int* ksplit,
                           hipStream_t s);
int z2z_launch_small_input(z2z_ctx* c, const void* A, const void* W, void* out, int R, const int32_t* rows_dev, int N, int K, const z2z_small_weight* weight,
                           hipStream_t s);
