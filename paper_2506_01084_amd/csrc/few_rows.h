// Products of a few rows in one launch with their epilogue (few_rows.hip): the gated block's first, F = act(X W[:d_ff]^T) * (X W[d_ff:]^T) with what the backward pass
// needs in `kept` where that names anything, and its second, out = X W^T + residual (f32: both fp32).  group: 0 = bf16 weights, else 4 bits.  K a multiple of 64, the
// weights' rows of 16.
#pragma once

#include "z2z_internal.h"

int z2z_launch_few_gated(const void* X, const void* W, const void* scale, int group, int act, void* F, const z2z_ffn_kept& kept, int R, const int32_t* rows_dev, int d_ff,
                         int K, hipStream_t s);
int z2z_launch_few_linear(const void* X, const void* W, const void* scale, int group, const void* residual, void* out, bool f32, int R, const int32_t* rows_dev,
                          int N, int K, hipStream_t s);
