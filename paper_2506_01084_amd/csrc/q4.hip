// Products of a few rows with 4-bit weights (gfx950): w[n, k] = scale[k / group, n] * v[n, k], v one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a sign (e2m1), scales bf16,
// group 32, 64 or 128.  A generation step through the learned hyper-encoder (zip2zip paper, section 2.2) is bound by the bytes of its weights; these are a
// quarter.
//
// Layout: blocks of 16 weight rows x 128 columns, 1024 bytes in the order in which the lanes of a wave take them: lane 16 j + r holds, in word m of its 16
// bytes, columns 32 m + 8 j .. + 7 of row r -- of each of the block's four matrix instructions (16 x 16 x 32) the eight it supplies.  The hardware turns a byte into
// two bf16, exactly; the products of a group are summed in fp32, and the scale multiplies the sum: nothing is rounded but sums.  (Whole numbers q - 8 made as 128 + q in
// bf16, with 136 times the sum of the rows' values taken off again, cost as much and leave the rounding of sums 136 times as large.)
// Rows beyond the last whole block of columns are filled up with zeros.
#include "q4.h"

#include <algorithm>

namespace {

using z2z_logits::bf16_bits_rne;
using z2z_logits::f32x4;
using z2z_q4::mfma;
using z2z_q4::values_of;

constexpr int Q_BLOCK = 128;             // columns of a block

// ---- bf16 -> 4 bits: a wave per block --------------------------------------------------------------------------------------------
// scale = largest magnitude of the group / 6, rounded to bf16; v = the nearest to w / scale, of two as near the one whose code is even.  (Where that changes is
// a product of the scale and a number of three bits: exact in fp32.  Magnitudes are compared by their bits, in which a NaN is the largest: a group that
// holds a NaN or an infinity has the scale NaN, and zeros.)
__global__ void __launch_bounds__(256) q4_quantize_kernel(const uint16_t* W, int cols, int chain, long long n_blocks, uint4* q, uint16_t* scale, int rows) {
  const int lane = threadIdx.x & 63, r = lane & 15, j = lane >> 4;
  const long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= n_blocks) return;
  const int kblocks = (cols + Q_BLOCK - 1) / Q_BLOCK;
  const long long n16 = id / kblocks;
  const int kb = (int)(id - n16 * kblocks);
  const uint16_t* row = W + (size_t)(n16 * 16 + r) * cols;
  uint4 v[4];
  uint32_t most[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int col = kb * Q_BLOCK + m * 32 + j * 8;
    v[m] = uint4{0u, 0u, 0u, 0u};
    if (col < cols) v[m] = *reinterpret_cast<const uint4*>(row + col);
    const uint32_t w[4] = {v[m].x, v[m].y, v[m].z, v[m].w};
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) a = max(a, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    a = max(a, (uint32_t)__shfl_xor((int)a, 16));
    most[m] = max(a, (uint32_t)__shfl_xor((int)a, 32));
  }
  if (chain >= 2) {
    most[0] = most[1] = max(most[0], most[1]);
    most[2] = most[3] = max(most[2], most[3]);
  }
  if (chain == 4) most[0] = most[1] = most[2] = most[3] = max(most[0], most[2]);
  uint32_t out[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int col = kb * Q_BLOCK + m * 32;
    const bool finite = most[m] < 0x7F80u;
    const uint32_t bits = finite ? bf16_bits_rne(__fdiv_rn(__uint_as_float(most[m] << 16), 6.0f)) : 0x7FC0u;
    const float s = __uint_as_float(bits << 16);
    const uint32_t w[4] = {v[m].x, v[m].y, v[m].z, v[m].w};
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
      const float y = fabsf(x);
      const int code = (y > 0.25f * s) + (y >= 0.75f * s) + (y > 1.25f * s) + (y >= 1.75f * s) + (y > 2.5f * s) + (y >= 3.5f * s) + (y > 5.f * s);
      if (finite && s > 0.f && code > 0) word |= (uint32_t)(code | (x < 0.f ? 8 : 0)) << (4 * i);
    }
    out[m] = col < cols ? word : 0u;
    if (j == 0 && m % chain == 0 && col < cols) scale[(size_t)(col / (32 * chain)) * rows + n16 * 16 + r] = (uint16_t)bits;
  }
  q[id * 64 + lane] = uint4{out[0], out[1], out[2], out[3]};
}

// ---- 4 bits -> bf16, each weight rounded once: for calls of many rows, whose products run on the tile kernel ----------------------------------
__global__ void __launch_bounds__(256) q4_expand_kernel(const uint4* q, const uint16_t* scale, int rows, int cols, int chain, long long n_blocks, uint16_t* W) {
  const int lane = threadIdx.x & 63, r = lane & 15, j = lane >> 4;
  const long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= n_blocks) return;
  const int kblocks = (cols + Q_BLOCK - 1) / Q_BLOCK;
  const long long n16 = id / kblocks;
  const int kb = (int)(id - n16 * kblocks);
  const uint4 words = q[id * 64 + lane];
  const uint32_t w[4] = {words.x, words.y, words.z, words.w};
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int col = kb * Q_BLOCK + m * 32 + j * 8;
    if (col >= cols) continue;
    const float s = __uint_as_float((uint32_t)scale[(size_t)(col / (32 * chain)) * rows + n16 * 16 + r] << 16);
    const uint4 p = values_of(w[m]);
    const uint32_t pair[4] = {p.x, p.y, p.z, p.w};
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      o[i] = z2z_logits::pack_bf16(__uint_as_float(pair[i] << 16) * s, __uint_as_float(pair[i] & 0xFFFF0000u) * s);
    *reinterpret_cast<uint4*>(W + (size_t)(n16 * 16 + r) * cols + col) = uint4{o[0], o[1], o[2], o[3]};
  }
}

// ---- the product ------------------------------------------------------------------------------------------------------------------
struct Q4Args {
  const uint4* q;
  const uint16_t* scale;   // [K / group, N]
  const uint16_t* X;       // [R, K]
  float* partial;          // [ksplit][R][N]
  int32_t R, N, K, kblocks, per;     // per: blocks of a part
  const int32_t* rows_dev;
};

constexpr int Q_WAVES = 4, Q_TILES = 2;              // a wave has Q_TILES tiles of 16 weight rows
constexpr int Q_ROWS = 16 * Q_TILES * Q_WAVES;       // weight rows of a workgroup
constexpr int Q_CHUNK = 256;                         // columns between two barriers
constexpr int Q_STEPS = Q_CHUNK / Q_BLOCK;

// Workgroup = 128 weight rows x a part of K x up to 16 NB rows of X.  X goes through LDS 256 columns at a time, in the order of the matrix instruction's operand
// (position r of a fragment's 16 exchanged by the column chunk, so that writes of consecutive chunks are on different banks), its scales beside it; the
// weights go from memory to registers, two chunks (8 loads of 1024 bytes a wave) ahead.  CHAIN: matrix instructions per group.  (512 columns a chunk, one
// ahead: 24 rows, d = 3584, d_ff = 9600 13.2 us instead of 11.9 for the first product, 9.2 instead of 8.9 for the second.)  Bounds on the waves of a SIMD keep the sums out of
// AGPRs, which the scaling would have to copy them from (300 rows, d = 2048, d_ff = 5504, groups of 32: the block 73 -> 65 us; d = 4096 178 -> 163).
template <int CHAIN, int NB>
__global__ void __launch_bounds__(64 * Q_WAVES, NB == 1 ? 4 : NB == 2 ? 3 : 2) q4_kernel(Q4Args a) {
  __shared__ uint4 xs[Q_CHUNK / 32 * NB * 64];
  __shared__ uint4 ss[Q_CHUNK / 32 / CHAIN * Q_ROWS / 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, j = lane >> 4;
  const int R = a.rows_dev ? min(a.R, *a.rows_dev) : a.R;
  const int row0 = (int)blockIdx.z * 16 * NB;
  if (row0 >= R) return;                             // (the whole workgroup)
  const int n_wg = (int)blockIdx.x * Q_ROWS;
  const int n0 = n_wg + wave * 16 * Q_TILES;
  const int b0 = (int)blockIdx.y * a.per, b1 = min(b0 + a.per, a.kblocks);
  const int groups = a.K / (32 * CHAIN);
  constexpr int XV = NB * Q_CHUNK / 8 * 16 / (64 * Q_WAVES);         // 16-byte pieces of X a thread moves per chunk
  constexpr int SV = (Q_CHUNK / 32 / CHAIN * Q_ROWS / 8 + 64 * Q_WAVES - 1) / (64 * Q_WAVES);
  uint4 xv[XV], sv[SV], w[2][Q_STEPS][Q_TILES];

  // (columns behind the part's end and rows that do not exist are zeros: what the weights there are read as does not count)
  auto fetch = [&](int blk) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < XV; ++v) {
      const int t = v * 64 * Q_WAVES + tid, c = t % (Q_CHUNK / 8), row = row0 + t / (Q_CHUNK / 8), col = blk * Q_BLOCK + c * 8;
      xv[v] = uint4{0u, 0u, 0u, 0u};
      if (row < R && col < min(b1 * Q_BLOCK, a.K)) xv[v] = *reinterpret_cast<const uint4*>(a.X + (size_t)row * a.K + col);
    }
#pragma unroll
    for (int v = 0; v < SV; ++v) {
      const int t = v * 64 * Q_WAVES + tid, n = n_wg + t % (Q_ROWS / 8) * 8, g = t / (Q_ROWS / 8), at = blk * (4 / CHAIN) + g;
      sv[v] = uint4{0u, 0u, 0u, 0u};
      if (g < Q_CHUNK / 32 / CHAIN && n < a.N && at < min(b1 * (4 / CHAIN), groups)) sv[v] = *reinterpret_cast<const uint4*>(a.scale + (size_t)at * a.N + n);
    }
  };
  auto publish = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < XV; ++v) {
      const int t = v * 64 * Q_WAVES + tid, c = t % (Q_CHUNK / 8), row = t / (Q_CHUNK / 8);
      xs[((c >> 2) * NB + (row >> 4)) * 64 + (c & 3) * 16 + ((row & 15) ^ (c & 15))] = xv[v];
    }
#pragma unroll
    for (int v = 0; v < SV; ++v) {
      const int t = v * 64 * Q_WAVES + tid;
      if (SV * 64 * Q_WAVES == Q_CHUNK / 32 / CHAIN * Q_ROWS / 8 || t < Q_CHUNK / 32 / CHAIN * Q_ROWS / 8) ss[t] = sv[v];
    }
  };
  auto fetch_w = [&](uint4 (&to)[Q_STEPS][Q_TILES], int blk) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < Q_STEPS; ++s)
#pragma unroll
      for (int t = 0; t < Q_TILES; ++t) {
        const size_t tile = (size_t)min((n0 >> 4) + t, (a.N >> 4) - 1);
        to[s][t] = a.q[(tile * a.kblocks + min(blk + s, b1 - 1)) * 64 + lane];
      }
  };

  f32x4 acc[Q_TILES][NB];
#pragma unroll
  for (int t = 0; t < Q_TILES; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

  auto compute = [&](const uint4 (&wc)[Q_STEPS][Q_TILES]) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < Q_STEPS; ++s) {
      f32x4 part[Q_TILES][NB];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const int k = s * 4 + m;
        uint4 x[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) x[b] = xs[(k * NB + b) * 64 + j * 16 + (r ^ ((k * 4 + j) & 15))];
#pragma unroll
        for (int t = 0; t < Q_TILES; ++t) {
          const uint4 words = wc[s][t];
          const uint4 p = values_of(m == 0 ? words.x : m == 1 ? words.y : m == 2 ? words.z : words.w);
#pragma unroll
          for (int b = 0; b < NB; ++b) part[t][b] = mfma(p, x[b], m % CHAIN == 0 ? zero : part[t][b]);
        }
        if (m % CHAIN == CHAIN - 1) {
#pragma unroll
          for (int t = 0; t < Q_TILES; ++t) {
            // (the lane's four rows of the tile)
            const uint2 s4 = reinterpret_cast<const uint2*>(ss)[k / CHAIN * (Q_ROWS / 4) + (wave * Q_TILES + t) * 4 + j];
            const float sc[4] = {__uint_as_float(s4.x << 16), __uint_as_float(s4.x & 0xFFFF0000u), __uint_as_float(s4.y << 16),
                                 __uint_as_float(s4.y & 0xFFFF0000u)};
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                acc[t][b][e] = fmaf(sc[e], part[t][b][e], acc[t][b][e]);
                asm volatile("" : "+v"(acc[t][b][e]));   // (here and now: else the sums of a chunk are all kept, and multiplied behind the next branch)
              }
          }
        }
      }
    }
  };

  // (The weights ahead are asked for behind the part's end, too, where they are its last block's, and there is no way out of the middle of the loop: where
  // loads may have been left out the compiler waits for all of them before it publishes the rows.)
  fetch_w(w[0], b0);
  __builtin_amdgcn_sched_barrier(0);
  fetch(b0);
  __builtin_amdgcn_sched_barrier(0);
  fetch_w(w[1], b0 + Q_STEPS);
  int blk = b0, chunks = (b1 - b0 + Q_STEPS - 1) / Q_STEPS;
  for (; chunks >= 2; chunks -= 2, blk += 2 * Q_STEPS) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      publish();
      __syncthreads();
      fetch(blk + (u + 1) * Q_STEPS);
      compute(w[u]);
      fetch_w(w[u], blk + (u + 2) * Q_STEPS);
      __syncthreads();
    }
  }
  if (chunks > 0) {
    publish();
    __syncthreads();
    compute(w[0]);
  }
  float* out = a.partial + (size_t)blockIdx.y * a.R * a.N;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int row = row0 + b * 16 + r;
#pragma unroll
    for (int t = 0; t < Q_TILES; ++t) {
      const int n = n0 + t * 16 + j * 4;
      if (row < R && n < a.N) *reinterpret_cast<float4*>(out + (size_t)row * a.N + n) = float4{acc[t][b][0], acc[t][b][1], acc[t][b][2], acc[t][b][3]};
    }
  }
}

template <int CHAIN>
void launch_q4(const Q4Args& a, dim3 grid, int blocks, hipStream_t s) {
  if (blocks == 1)
    hipLaunchKernelGGL((q4_kernel<CHAIN, 1>), grid, dim3(64 * Q_WAVES), 0, s, a);
  else if (blocks == 2)
    hipLaunchKernelGGL((q4_kernel<CHAIN, 2>), grid, dim3(64 * Q_WAVES), 0, s, a);
  else if (blocks == 3)
    hipLaunchKernelGGL((q4_kernel<CHAIN, 3>), grid, dim3(64 * Q_WAVES), 0, s, a);
  else
    hipLaunchKernelGGL((q4_kernel<CHAIN, 4>), grid, dim3(64 * Q_WAVES), 0, s, a);
}

long long blocks_of(int rows, int cols) { return (long long)(rows / 16) * ((cols + Q_BLOCK - 1) / Q_BLOCK); }

}  // namespace

int z2z_launch_quantize_q4(const void* W, int rows, int cols, int group, void* q, void* scale, hipStream_t s) {
  const long long n = blocks_of(rows, cols);
  if ((n + 3) / 4 * 256 > kLaunchThreads) return Z2Z_EUNSUPPORTED;
  hipLaunchKernelGGL(q4_quantize_kernel, dim3((unsigned)((n + 3) / 4)), dim3(256), 0, s, reinterpret_cast<const uint16_t*>(W), cols, group / 32, n,
                     reinterpret_cast<uint4*>(q), reinterpret_cast<uint16_t*>(scale), rows);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

int z2z_launch_expand_q4(const void* q, const void* scale, int rows, int cols, int group, void* W, hipStream_t s) {
  const long long n = blocks_of(rows, cols);
  if ((n + 3) / 4 * 256 > kLaunchThreads) return Z2Z_EUNSUPPORTED;
  hipLaunchKernelGGL(q4_expand_kernel, dim3((unsigned)((n + 3) / 4)), dim3(256), 0, s, reinterpret_cast<const uint4*>(q),
                     reinterpret_cast<const uint16_t*>(scale), rows, cols, group / 32, n, reinterpret_cast<uint16_t*>(W));
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

int z2z_launch_q4_parts(z2z_ctx* c, const void* X, const void* q, const void* scale, int group, int R, const int32_t* rows_dev, int N, int K,
                        const float** partial, int* ksplit, hipStream_t s) {
  Q4Args a;
  a.q = reinterpret_cast<const uint4*>(q);
  a.scale = reinterpret_cast<const uint16_t*>(scale);
  a.X = reinterpret_cast<const uint16_t*>(X);
  a.R = R;
  a.N = N;
  a.K = K;
  a.rows_dev = rows_dev;
  a.kblocks = (K + Q_BLOCK - 1) / Q_BLOCK;
  // rows go in equal runs of up to 64; parts of K for as many workgroups as are there at a time, with as many registers as the rows take
  const int runs = (R + 63) / 64, blocks = ((R + runs - 1) / runs + 15) / 16;
  const int tiles = (N + Q_ROWS - 1) / Q_ROWS, most = (a.kblocks + Q_STEPS - 1) / Q_STEPS;
  const int target = c->num_cu * (blocks == 1 ? 5 : blocks == 2 ? 4 : 3) / 2;
  const int ways = std::max(1, std::min(target / (tiles * runs), most));
  a.per = (a.kblocks + ways - 1) / ways;
  a.per = std::min((a.per + Q_STEPS - 1) / Q_STEPS * Q_STEPS, a.kblocks);
  *ksplit = (a.kblocks + a.per - 1) / a.per;
  float* p = nullptr;
  const int rc = z2z_partial_reserve(c, (size_t)*ksplit * R * N * sizeof(float), &p, s);
  if (rc != Z2Z_OK) return rc;
  a.partial = p;
  *partial = p;
  const dim3 grid((unsigned)tiles, (unsigned)*ksplit, (unsigned)((R + 16 * blocks - 1) / (16 * blocks)));
  if (group == 32)
    launch_q4<1>(a, grid, blocks, s);
  else if (group == 64)
    launch_q4<2>(a, grid, blocks, s);
  else
    launch_q4<4>(a, grid, blocks, s);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}
