// The gated feed-forward block's two products for a few rows (gfx950), each in one launch with its epilogue: F = act(X Wg^T) * (X Wu^T), then Y = F W2^T + residual,
// over weights in bf16 or in 4 bits (q4.hip says how these lie).
//
// Bound by the weights' bytes, and where those are few by round trips: so nothing is split over workgroups and added up by a launch of its own.  A workgroup
// takes TILES x 16 weight rows (a gated product: 16 gate rows and the same 16 of the other projection) over all of K; its waves share K out, each
// streams its own part from memory to registers in the order of the matrix instruction's operand, the rows' values beside it, and the waves' sums meet in LDS,
// in order.  K goes in units of 128 columns, the loads of the next ones ahead of the arithmetic on these.
#include "few_rows.h"

#include "gated.h"
#include "q4.h"

#include <algorithm>

namespace {

using z2z_logits::f32x4;
using z2z_logits::load_if;
using z2z_q4::mfma;
using z2z_q4::values_of;

constexpr int W_UNIT = 128;              // columns

struct FewArgs {
  const unsigned char* W;
  const uint16_t* scale;   // 4 bits: [K / group, n_w]
  const uint16_t* X;       // [R, K]
  void* out;               // gated: F [R, N] bf16; else [R, N] bf16 or fp32
  const void* residual;    // else: [R, N] as `out`, or nullptr
  z2z_ffn_kept kept;       // gated: what the backward pass is given, or nothing
  const int32_t* rows_dev;
  int32_t R, N, K, n_w;    // n_w: rows of W
  int32_t act, f32;
};

__device__ __forceinline__ uint32_t word_of(const uint4& v, int m) { return m == 0 ? v.x : m == 1 ? v.y : m == 2 ? v.z : v.w; }

// WAVES: of a workgroup, that share K out.  CHAIN: 0 = bf16 weights, else 4 bits with a scale per CHAIN matrix instructions (of 32 columns); TILES: tiles of 16 weight rows; NB: blocks of 16 rows of X.
template <int W_WAVES, int CHAIN, int TILES, int NB, bool GATED>
__global__ void __launch_bounds__(64 * W_WAVES, 2) few_rows_kernel(FewArgs a) {
  constexpr bool Q4 = CHAIN != 0;
  constexpr int LOADS = Q4 ? 1 : 4;                // of a tile's unit, 16 bytes a lane
  constexpr int SCALES = Q4 ? 4 / (Q4 ? CHAIN : 1) : 1;
  constexpr int DEPTH = Q4 && NB == 1 ? 2 : 1;     // units ahead (three of weights with one of X: 1 row, d = 4096, d_ff = 10944 19.8 us -> 23.2)
  __shared__ f32x4 sums[W_WAVES][TILES * NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r = lane & 15, j = lane >> 4;
  const int R = a.rows_dev ? min(a.R, *a.rows_dev) : a.R;
  const int row0 = (int)blockIdx.y * 16 * NB;
  if (row0 >= R) return;                           // (the whole workgroup)
  // first weight row of every tile, and of the outputs
  int first[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) first[t] = GATED ? ((int)blockIdx.x * (TILES / 2) + (t >> 1)) * 16 + (t & 1) * a.N : ((int)blockIdx.x * TILES + t) * 16;
  const int units = (a.K + W_UNIT - 1) / W_UNIT, per = (units + W_WAVES - 1) / W_WAVES;
  const int u0 = wave * per, u1 = min(u0 + per, units);

  const unsigned char* w_at[TILES];
  const uint16_t* s_at[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int n0 = min(first[t], a.n_w - 16);
    w_at[t] = Q4 ? a.W + ((size_t)(n0 >> 4) * units * 64 + lane) * 16 : a.W + ((size_t)(n0 + r) * a.K + j * 8) * 2;
    s_at[t] = Q4 ? a.scale + n0 + j * 4 : nullptr;
  }
  const uint16_t* x_at[NB];
  bool x_ok[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int row = row0 + b * 16 + r;
    x_ok[b] = row < R;
    x_at[b] = a.X + (size_t)min(row, R - 1) * a.K + j * 8;
  }

  struct Unit {
    uint4 w[TILES][LOADS];
    uint2 s[TILES][SCALES];
    uint4 x[NB][4];
  };
  // (columns behind the last, where a unit's second half is not there: zeros of X, and of bf16 weights before they are multiplied, which may be infinite where they are read)
  auto fetch = [&](Unit& f, int u) __attribute__((always_inline)) {
    const bool whole = (u + 1) * W_UNIT <= a.K;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      if (Q4) {
        f.w[t][0] = *reinterpret_cast<const uint4*>(w_at[t] + (size_t)u * 1024);
#pragma unroll
        for (int g = 0; g < SCALES; ++g) {
          f.s[t][g] = uint2{0u, 0u};
          if (whole || g * CHAIN * 32 < W_UNIT / 2) f.s[t][g] = *reinterpret_cast<const uint2*>(s_at[t] + (size_t)(u * SCALES + g) * a.n_w);
        }
      } else {
#pragma unroll
        for (int l = 0; l < LOADS; ++l) f.w[t][l] = *reinterpret_cast<const uint4*>(w_at[t] + (size_t)u * (2 * W_UNIT) + (whole || l < 2 ? l : 0) * 64);
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int m = 0; m < 4; ++m) f.x[b][m] = load_if(x_ok[b] && (whole || m < 2), reinterpret_cast<const uint4*>(x_at[b] + u * W_UNIT + m * 32));
  };

  f32x4 acc[TILES][NB];
#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto compute = [&](const Unit& f, int u) __attribute__((always_inline)) {
    const uint32_t second = Q4 || (u + 1) * W_UNIT <= a.K ? 0xFFFFFFFFu : 0u;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      f32x4 part[NB];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        uint4 v = Q4 ? values_of(word_of(f.w[t][0], m)) : f.w[t][Q4 ? 0 : m];
        if (!Q4 && m >= 2) v = uint4{v.x & second, v.y & second, v.z & second, v.w & second};
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if (Q4)
            part[b] = mfma(v, f.x[b][m], m % (Q4 ? CHAIN : 1) == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : part[b]);
          else
            acc[t][b] = mfma(v, f.x[b][m], acc[t][b]);
        }
        if (Q4 && m % (Q4 ? CHAIN : 1) == (Q4 ? CHAIN : 1) - 1) {
          const uint2 s = f.s[t][m / (Q4 ? CHAIN : 1)];
          const float sc[4] = {__uint_as_float(s.x << 16), __uint_as_float(s.x & 0xFFFF0000u), __uint_as_float(s.y << 16),
                               __uint_as_float(s.y & 0xFFFF0000u)};
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              acc[t][b][e] = fmaf(sc[e], part[b][e], acc[t][b][e]);
              asm volatile("" : "+v"(acc[t][b][e]));     // (here and now, not behind the next branch with all parts kept)
            }
        }
      }
    }
  };

  // units u0 .. u1 - 1, DEPTH + 1 of them in registers
  Unit f[DEPTH + 1];
#pragma unroll
  for (int k = 0; k < DEPTH; ++k)
    if (u0 + k < u1) fetch(f[k], u0 + k);
  for (int u = u0; u < u1; u += DEPTH + 1) {
#pragma unroll
    for (int k = 0; k <= DEPTH; ++k) {
      if (u + k + DEPTH < u1) fetch(f[(k + DEPTH) % (DEPTH + 1)], u + k + DEPTH);
      if (u + k < u1) compute(f[k], u + k);
    }
  }

#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) sums[wave][t * NB + b][lane] = acc[t][b];
  __syncthreads();
  // a thread's piece: 4 columns of a row.  Pieces of a tile (GATED: of a pair of tiles) and block: 64
  constexpr int PIECES = (GATED ? TILES / 2 : TILES) * NB * 64;
  for (int p = threadIdx.x; p < PIECES; p += 64 * W_WAVES) {
    const int l = p & 63, b = (p >> 6) % NB, t = (p >> 6) / NB;
    const int row = row0 + b * 16 + (l & 15), n = ((int)blockIdx.x * (GATED ? TILES / 2 : TILES) + t) * 16 + (l >> 4) * 4;
    if (row >= R || n >= a.N) continue;
    if (GATED) {
      float g[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W_WAVES; ++w) {
        const f32x4 x = sums[w][2 * t * NB + b][l], y = sums[w][(2 * t + 1) * NB + b][l];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          g[e] += x[e];
          u[e] += y[e];
        }
      }
      const size_t e = (size_t)row * a.N + n;
      uint2* f4 = reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + e);
      *f4 = z2z_gated::hidden_and_keep4(g, u, a.act, a.kept, e);
    } else {
      float4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W_WAVES; ++w) {
        const f32x4 y = sums[w][t * NB + b][l];
        x = float4{x.x + y[0], x.y + y[1], x.z + y[2], x.w + y[3]};
      }
      z2z_logits::finish_linear(x, float4{0.f, 0.f, 0.f, 0.f}, 0, a.residual, a.out, a.f32, (size_t)row * a.N + n);
    }
  }
}

// (a gated product has enough workgroups for four waves each, of which more fit a CU: 1 row, 4 bits, d = 4096, d_ff = 10944 16.9 -> 14.2 us, 16 rows 21.4 -> 18.5;
// the second one's 256 take eight: 7.9 us, 10.5 with four.)
template <int CHAIN, int TILES, bool GATED>
void launch(const FewArgs& a, int tiles, int blocks, hipStream_t s) {
  const dim3 grid((unsigned)tiles, (unsigned)((a.R + 16 * blocks - 1) / (16 * blocks)));
  constexpr int WAVES = GATED ? 4 : 8;
  if (blocks == 1)
    hipLaunchKernelGGL((few_rows_kernel<WAVES, CHAIN, TILES, 1, GATED>), grid, dim3(64 * WAVES), 0, s, a);
  else if (blocks == 2)
    hipLaunchKernelGGL((few_rows_kernel<WAVES, CHAIN, TILES, 2, GATED>), grid, dim3(64 * WAVES), 0, s, a);
  else
    hipLaunchKernelGGL((few_rows_kernel<WAVES, CHAIN, TILES, 4, GATED>), grid, dim3(64 * WAVES), 0, s, a);
}

// Blocks of 16 rows a workgroup takes: runs of equal length, of up to 64 rows.
int few_blocks(int R) {
  const int runs = (R + 63) / 64, blocks = ((R + runs - 1) / runs + 15) / 16;
  return blocks <= 2 ? blocks : 4;
}

template <int TILES, bool GATED>
void launch_group(const FewArgs& a, int group, int tiles, int blocks, hipStream_t s) {
  if (group == 0)
    launch<0, TILES, GATED>(a, tiles, blocks, s);
  else if (group == 32)
    launch<1, TILES, GATED>(a, tiles, blocks, s);
  else if (group == 64)
    launch<2, TILES, GATED>(a, tiles, blocks, s);
  else
    launch<4, TILES, GATED>(a, tiles, blocks, s);
}

}  // namespace

int z2z_launch_few_gated(const void* X, const void* W, const void* scale, int group, int act, void* F, const z2z_ffn_kept& kept, int R, const int32_t* rows_dev, int d_ff,
                         int K, hipStream_t s) {
  const FewArgs a = {reinterpret_cast<const unsigned char*>(W), reinterpret_cast<const uint16_t*>(scale), reinterpret_cast<const uint16_t*>(X), F, nullptr,
                     kept, rows_dev, R, d_ff, K, 2 * d_ff, act, 0};
  launch_group<2, true>(a, group, d_ff / 16, few_blocks(R), s);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

int z2z_launch_few_linear(const void* X, const void* W, const void* scale, int group, const void* residual, void* out, bool f32, int R, const int32_t* rows_dev,
                          int N, int K, hipStream_t s) {
  const FewArgs a = {reinterpret_cast<const unsigned char*>(W), reinterpret_cast<const uint16_t*>(scale), reinterpret_cast<const uint16_t*>(X), out, residual,
                     z2z_ffn_kept{}, rows_dev, R, N, K, N, 0, f32 ? 1 : 0};
  launch_group<1, false>(a, group, N / 16, few_blocks(R), s);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}
