// sum[r] = sum_k weight[r, k] W[ids[r, k]] over the columns that a row lists, W the joint unembedding [W_base ; W_hyper[b]]: the listed part of
// the distillation loss's gradient with respect to the hidden rows, which the products of the other columns are added to.
#pragma once

#include "logits_common.h"

namespace z2z_listed {

struct ListedArgs {
  const int32_t* ids;       // [rows, K]
  const float* weight;      // [rows, K]
  const int32_t* size;      // [sequences]
  const uint4 *W_base, *W_hyper;
  float4* sum;              // [rows, d]
  int32_t rows, rows_per_seq, V, cap, K;
  int32_t n_chunks, slices; // 16-byte pieces of a row, and those by 64
};

// One wave, 64 pieces of 16 bytes of row r = wid / slices: eight rows of W requested at a time; fp32.
__device__ __forceinline__ void add_listed_rows(const ListedArgs& a, long long wid) {
  const int lane = threadIdx.x & 63;
  const int r = (int)(wid / a.slices);
  if (r >= a.rows) return;
  const int chunk = (int)(wid % a.slices) * 64 + lane;
  const int b = r / a.rows_per_seq;
  const int columns = a.V + min(max(a.size[b], 0), a.cap);
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  for (int k0 = 0; k0 < a.K; k0 += 64) {
    const int k = k0 + lane;
    const int my_id = k < a.K ? a.ids[(size_t)r * a.K + k] : -1;
    const float my_w = k < a.K && my_id >= 0 && my_id < columns ? a.weight[(size_t)r * a.K + k] : 0.f;
    uint64_t left = __ballot(my_w != 0.f);
    while (left != 0ull) {
      uint4 x[8];
      float w[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int l = left != 0ull ? __ffsll((long long)left) - 1 : 0;
        const int id = __builtin_amdgcn_readlane(my_id, l);
        w[u] = left != 0ull ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(my_w), l)) : 0.f;
        const bool there = left != 0ull;
        const uint4* row = !there ? a.W_base
                                  : (id < a.V ? a.W_base + (size_t)id * a.n_chunks : a.W_hyper + ((size_t)b * a.cap + (id - a.V)) * a.n_chunks);
        x[u] = there ? row[min(chunk, a.n_chunks - 1)] : uint4{0u, 0u, 0u, 0u};
        left &= left - 1ull;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const uint32_t xs[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[2 * e] = fmaf(w[u], __uint_as_float(xs[e] << 16), acc[2 * e]);
          acc[2 * e + 1] = fmaf(w[u], __uint_as_float(xs[e] & 0xFFFF0000u), acc[2 * e + 1]);
        }
      }
    }
  }
  if (chunk >= a.n_chunks) return;
  float4* to = a.sum + ((size_t)r * a.n_chunks + chunk) * 2;
  to[0] = float4{acc[0], acc[1], acc[2], acc[3]};
  to[1] = float4{acc[4], acc[5], acc[6], acc[7]};
}

}  // namespace z2z_listed
