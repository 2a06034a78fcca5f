// Products of the gated feed-forward block with fewer output tiles of 256 x 256 than the chip has CUs (gfx950, bf16): the tile kernel leaves most of the CUs without one then, and
// those it has wait for memory at every slab (logits_fast.hip).  Here a tile is 64 x 64 and a workgroup small enough that several share a CU and wait in turn.
//
// Workgroup = 4 waves, 2 x 2, of 32 weight rows ("A") x 32 rows of H ("B") each: 2 x 2 blocks of v_mfma_f32_16x16x32_bf16.  K goes in slabs of 64; a slab's two operand tiles, 8 KiB
// each, go through registers, two slabs ahead, into one of two LDS buffers: one barrier a slab.  Either operand is K-minor ([rows, K]: a row is 128 bytes, its 16-byte
// chunk c at c ^ (row & 7)) or K-major ([K, rows]: 64 rows of 128 bytes, read transposed; the 32-byte piece b of row k at b ^ g(k), g = bits 1 and 3 of k, so that
// the eight pieces that 32 lanes read at a time are on different banks).  A lane's two blocks of weight rows are groups of four that alternate, so that it stores eight columns
// of a row at once (the gated product: the gate's block and the other projection's); the places in LDS follow.  Widths are multiples of 64: only the rows of the call have a ragged end.
// Bound by LDS reads (32 KB a slab for 128 clocks of matrix instructions), half of the peak at best, and at these sizes by launches and round trips: products that do not
// need each other share a launch (forward and gradient, d = 1024, d_ff = 2752: 237 rows 67 -> 57 us, 1000 rows 141 -> 126; d = 256, d_ff = 704, 237 rows 34 -> 25).
// 237 rows, d = 1024, d_ff = 2752, each in a launch of its own (us, / on the kernels for more or fewer rows): first product 13.1 / 21.1, second 10.0 with its sum / 15.4, dF 10.9 / 28,
// dW2 and dW1 20.7 / 31, dX 13.9 with its sum / 31.
#include "small_tile.h"

#include "gated.h"

#include <algorithm>

namespace {

using z2z_logits::bf16x8;
using z2z_logits::f32x4;

constexpr int S_T = 64;                      // tile edge and slab
constexpr int S_D = 2;                       // slabs on their way in registers (forward and gradient, 237 rows, d = 1024, d_ff = 2752 57 us with one, 55 with two; four do not fit)
constexpr int S_WAVES = 4;                   // a SIMD: no accumulators in AGPRs

struct SmallArgs {
  const uint16_t *H, *W;
  void* out;
  const void* residual;
  float* partial;                            // [parts][R][N]
  z2z_ffn_kept kept;
  const int32_t *rows_dev, *k_dev;           // nullptr, or how many rows of the output, of the contraction, exist
  int32_t R, N, K, ldh, ldw, ldo;
  int32_t per;                               // slabs of a part
  int32_t tiles_n, tiles_r, n_work;
  int32_t d_ff, act, f32;
};

__device__ __forceinline__ uint2 read_transposed(const unsigned char* p) {
  typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
  typedef __attribute__((address_space(3))) s16x4* lds_ptr;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p));
}

__device__ __forceinline__ int piece_of(int k) { return ((k >> 1) & 1) | ((k >> 3) & 1) << 1; }

// Where chunk c of row t of an operand's 64 rows lies.
template <bool MAJOR, bool WIDE>
__device__ __forceinline__ int place(int t, int c) {
  if (!MAJOR) return t * 128 + ((c ^ (WIDE ? (t & 3) | ((t >> 3) & 1) << 2 : t & 7)) << 4);
  return t * 128 + (WIDE ? (c ^ (piece_of(t) >> 1) << 2) << 4 : (((c >> 1) ^ piece_of(t)) << 5) + ((c & 1) << 4));
}

template <bool MAJOR>
__device__ __forceinline__ uint4 in_order(const unsigned char* tile, int first, int q, int lane) {
  const int lane15 = lane & 15, quarter = lane >> 4;
  if (!MAJOR) return *reinterpret_cast<const uint4*>(tile + place<false, false>(first + lane15, 4 * q + quarter));
  const int k = 32 * q + 8 * quarter + (lane15 >> 2), at = (first >> 3) + ((lane & 3) >> 1), part = (lane & 1) * 8;
  const uint2 lo = read_transposed(tile + place<true, false>(k, at) + part), hi = read_transposed(tile + place<true, false>(k + 4, at) + part);
  return uint4{lo.x, lo.y, hi.x, hi.y};
}

// TW, TH: the operand is K-major.  EPI: 0 = out = sum + residual, 1 = the gated block's first product (a tile's 64 weight rows: 16 gate rows, 16 of the other
// projection, and once more), 2 = its gradient's.  PARTS: K is shared out over workgroups, and the sums of a part go to `partial` as they are.
template <bool TW, bool TH, int EPI, bool PARTS>
__device__ __forceinline__ void small_tile(const SmallArgs& a, unsigned block, unsigned char (&lds)[2][2][S_T * 128]) {
  constexpr bool WIDE = EPI != 1;             // a lane has 8 columns of a row in a row, not 4 of each of two blocks
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wv = wave & 1, wr = wave >> 1;
  const int lane15 = lane & 15, quarter = lane >> 4;
  // workgroup ids go round the 8 XCDs: an XCD takes a run of items, the tiles of a weight tile's rows next to each other
  const int each = (a.n_work + 7) / 8, item = (int)(block & 7) * each + (int)(block >> 3);
  if (item >= a.n_work || (int)(block >> 3) >= each) return;
  const int rt = item % a.tiles_r, rest = item / a.tiles_r, nt = rest % a.tiles_n, part = PARTS ? rest / a.tiles_n : 0;
  const int R = !TH && a.rows_dev ? min(a.R, max(__builtin_amdgcn_readfirstlane(*a.rows_dev), 0)) : a.R;
  const int r0 = rt * S_T;
  if (r0 >= R) return;
  const int k_rows = TH && a.k_dev ? min(a.K, max(__builtin_amdgcn_readfirstlane(*a.k_dev), 0)) : a.K;
  const int slabs = (k_rows + S_T - 1) / S_T;
  const int s0 = PARTS ? part * a.per : 0, s1 = PARTS ? min(s0 + a.per, slabs) : slabs;

  // ---- what a thread moves of a slab: rows tid / 8 and 32 more of either operand's 64, 16 bytes at chunk tid % 8
  const int row8 = tid >> 3, chunk = tid & 7;
  auto weight_row = [&](int t) { return EPI == 1 ? nt * 32 + (t >> 5) * 16 + (t & 15) + ((t >> 4) & 1) * a.d_ff : nt * S_T + t; };
  const uint16_t *w_at[2], *h_at[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = row8 + 32 * i;
    w_at[i] = TW ? a.W + nt * S_T + chunk * 8 : a.W + (size_t)weight_row(t) * a.ldw + chunk * 8;
    h_at[i] = TH ? a.H + r0 + chunk * 8 : a.H + (size_t)min(r0 + t, R - 1) * a.ldh + chunk * 8;
  }
  uint4 ahead[S_D][4];
  auto fetch = [&](uint4 (&v)[4], int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = min(s * S_T + row8 + 32 * i, k_rows - 1);
      v[i] = *reinterpret_cast<const uint4*>(w_at[i] + (TW ? (size_t)k * a.ldw : (size_t)s * S_T));
      v[2 + i] = *reinterpret_cast<const uint4*>(h_at[i] + (TH ? (size_t)k * a.ldh : (size_t)s * S_T));
    }
  };
  auto put = [&](int buf, const uint4 (&v)[4], int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = row8 + 32 * i;
      uint4 w = v[i], h = v[2 + i];
      if (TH && s * S_T + t >= k_rows) w = h = uint4{0u, 0u, 0u, 0u};      // (rows that do not exist: zeros on both sides)
      *reinterpret_cast<uint4*>(lds[buf][0] + place<TW, WIDE>(t, chunk)) = WIDE && TW && (piece_of(t) & 1) ? uint4{w.z, w.w, w.x, w.y} : w;
      *reinterpret_cast<uint4*>(lds[buf][1] + place<TH, false>(t, chunk)) = h;
    }
  };
  // fragments, k-step q of the slab: rows of the operand's 64 from `first`, 16 in order, or (WIDE) groups of four, every other one of 32
  auto weights_of = [&](int buf, int i, int q) __attribute__((always_inline)) -> uint4 {
    const unsigned char* tile = lds[buf][0];
    if (!WIDE) return in_order<TW>(tile, wv * 32 + i * 16, q, lane);
    if (!TW) return *reinterpret_cast<const uint4*>(tile + place<false, true>(wv * 32 + (lane15 >> 2) * 8 + i * 4 + (lane & 3), 4 * q + quarter));
    const int k = 32 * q + 8 * quarter + (lane15 >> 2), half = (i ^ (piece_of(k) & 1)) * 8;                                 // (rows k and k + 4 lie alike)
    const uint2 lo = read_transposed(tile + place<true, true>(k, wv * 4 + (lane & 3)) + half), hi = read_transposed(tile + place<true, true>(k + 4, wv * 4 + (lane & 3)) + half);
    return uint4{lo.x, lo.y, hi.x, hi.y};
  };

  f32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // one barrier: what a slab later goes to this buffer again is written behind the next one, which a wave reaches when it has read this
  auto multiply = [&](int buf) __attribute__((always_inline)) {
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      uint4 av[2], bv[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        av[i] = weights_of(buf, i, q);
        bv[i] = in_order<TH>(lds[buf][1], wr * 32 + i * 16, q, lane);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av[i]), __builtin_bit_cast(bf16x8, bv[j]), acc[i][j], 0, 0, 0);
    }
  };
  if (s0 < s1) {
#pragma unroll
    for (int u = 0; u < S_D; ++u) {
      fetch(ahead[u], min(s0 + u, s1 - 1));
      __builtin_amdgcn_sched_barrier(0);       // (in this order: the loop waits for the first slab's loads alone, not for what came behind them)
    }
    // (no way out of the middle of the loop: where loads may have been left out the compiler waits for all)
    int s = s0;
    for (; s + S_D <= s1; s += S_D) {
#pragma unroll
      for (int u = 0; u < S_D; ++u) {
        put(u & 1, ahead[u], s + u);
        fetch(ahead[u], min(s + u + S_D, s1 - 1));
        multiply(u & 1);
      }
    }
#pragma unroll
    for (int u = 0; u < S_D - 1; ++u) {
      if (s + u < s1) {
        put(u & 1, ahead[u], s + u);
        multiply(u & 1);
      }
    }
  }

  // ---- a lane has 4 columns of a row in each block
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = r0 + wr * 32 + j * 16 + lane15;
    if (row >= R) continue;
    if (EPI == 1) {
      const float g[4] = {acc[0][j][0], acc[0][j][1], acc[0][j][2], acc[0][j][3]}, u[4] = {acc[1][j][0], acc[1][j][1], acc[1][j][2], acc[1][j][3]};
      const int col = nt * 32 + wv * 16 + quarter * 4;
      const size_t at = (size_t)row * a.d_ff + col;
      uint2* f4 = reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + at);
      *f4 = z2z_gated::hidden_and_keep4(g, u, a.act, a.kept, at);
      continue;
    }
    const int col = nt * S_T + wv * 32 + quarter * 8;
    const float4 x0 = {acc[0][j][0], acc[0][j][1], acc[0][j][2], acc[0][j][3]}, x1 = {acc[1][j][0], acc[1][j][1], acc[1][j][2], acc[1][j][3]};
    if (PARTS) {
      float4* to = reinterpret_cast<float4*>(a.partial + ((size_t)part * a.R + row) * a.N + col);
      to[0] = x0;
      to[1] = x1;
    } else if (EPI == 2) {
      const size_t at = (size_t)row * a.d_ff + col;
      const float df0[4] = {x0.x, x0.y, x0.z, x0.w}, df1[4] = {x1.x, x1.y, x1.z, x1.w};
      const uint4* hi = reinterpret_cast<const uint4*>(a.kept.hi + at);
      const uint4 lo = *reinterpret_cast<const uint4*>(a.kept.lo + at);
      const z2z_gated::Slopes4 s0 = z2z_gated::slopes4(df0, hi[0], uint2{lo.x, lo.y}), s1 = z2z_gated::slopes4(df1, hi[1], uint2{lo.z, lo.w});
      uint16_t* to = reinterpret_cast<uint16_t*>(a.out) + (size_t)row * a.ldo + col;
      *reinterpret_cast<uint4*>(to) = uint4{s0.dg.x, s0.dg.y, s1.dg.x, s1.dg.y};
      *reinterpret_cast<uint4*>(to + a.d_ff) = uint4{s0.du.x, s0.du.y, s1.du.x, s1.du.y};
    } else {
      const size_t at = (size_t)row * a.ldo + col;
      if (a.f32) {
        z2z_logits::finish_linear(x0, float4{0.f, 0.f, 0.f, 0.f}, 0, a.residual, a.out, 1, at);
        z2z_logits::finish_linear(x1, float4{0.f, 0.f, 0.f, 0.f}, 0, a.residual, a.out, 1, at + 4);
        continue;
      }
      float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
      uint32_t r[4] = {0u, 0u, 0u, 0u};
      if (a.residual) {
        const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.residual) + at);
        r[0] = v.x, r[1] = v.y, r[2] = v.z, r[3] = v.w;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += __builtin_bit_cast(float, e & 1 ? r[e >> 1] & 0xffff0000u : r[e >> 1] << 16);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = z2z_logits::pack_bf16(x[2 * e], x[2 * e + 1]);
      *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(a.out) + at) = uint4{r[0], r[1], r[2], r[3]};
    }
  }
}

template <bool TW, int EPI, bool PARTS>
__global__ void __launch_bounds__(256, S_WAVES) small_tile_kernel(SmallArgs a) {
  __shared__ __align__(256) unsigned char lds[2][2][S_T * 128];
  small_tile<TW, false, EPI, PARTS>(a, blockIdx.x, lds);
}

// Two products that do not need each other in one launch: dF, or dX, in the first `n_a` workgroups, a weight gradient in the others.
template <int EPI, bool PARTS, bool W_PARTS>
__global__ void __launch_bounds__(256, S_WAVES) small_pair_kernel(SmallArgs a, SmallArgs b, unsigned n_a) {
  __shared__ __align__(256) unsigned char lds[2][2][S_T * 128];
  if (blockIdx.x < n_a)
    small_tile<true, false, EPI, PARTS>(a, blockIdx.x, lds);
  else
    small_tile<true, true, 0, W_PARTS>(b, blockIdx.x - n_a, lds);
}

// Parts of K for `tiles` tiles: as many as bring the workgroups up to `most`, of `least` slabs or more.
int cut(SmallArgs& a, int tiles, int most, int least) {
  const int slabs = (a.K + S_T - 1) / S_T, ways = std::max(1, std::min(most / std::max(tiles, 1), slabs / least));
  a.per = (slabs + ways - 1) / ways;
  return (slabs + a.per - 1) / a.per;
}
size_t part_bytes(const SmallArgs& a, int parts) { return parts > 1 ? (size_t)parts * a.R * a.N * sizeof(float) : 0; }

// The parts' buffers, behind each other.  b: nullptr, or a weight gradient beside `a`.
int reserve(z2z_ctx* c, SmallArgs& a, int parts, SmallArgs* b, int parts_b, hipStream_t s) {
  const size_t n = part_bytes(a, parts), m = b ? part_bytes(*b, parts_b) : 0;
  if (n + m == 0) return Z2Z_OK;
  float* p = nullptr;
  const int rc = z2z_partial_reserve(c, n + m, &p, s);
  a.partial = p;
  if (b) b->partial = p + n / sizeof(float);
  return rc;
}

int add_up(const SmallArgs& a, int parts, hipStream_t s) {
  return parts > 1 ? z2z_launch_linear_sum(a.partial, parts, a.R, a.rows_dev, a.N, a.residual, a.out, a.f32 != 0, s) : Z2Z_OK;
}

unsigned count(SmallArgs& a, int parts) {
  a.tiles_r = (a.R + S_T - 1) / S_T;
  a.n_work = a.tiles_r * a.tiles_n * parts;
  return (unsigned)((a.n_work + 7) / 8 * 8);
}

template <bool TW, int EPI, bool PARTS>
int launch(SmallArgs& a, int parts, hipStream_t s) {
  const unsigned n = count(a, parts);
  hipLaunchKernelGGL((small_tile_kernel<TW, EPI, PARTS>), dim3(n), dim3(256), 0, s, a);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

template <int EPI, bool PARTS>
int launch_pair(SmallArgs& a, int parts, SmallArgs& b, int parts_b, hipStream_t s) {
  const unsigned n_a = count(a, parts), n_b = count(b, parts_b);
  if (parts_b > 1)
    hipLaunchKernelGGL((small_pair_kernel<EPI, PARTS, true>), dim3(n_a + n_b), dim3(256), 0, s, a, b, n_a);
  else
    hipLaunchKernelGGL((small_pair_kernel<EPI, PARTS, false>), dim3(n_a + n_b), dim3(256), 0, s, a, b, n_a);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

int rows_of_tiles(int R) { return (R + S_T - 1) / S_T; }

// A product [R, N] whose tiles are fewer than the workgroups that the chip holds has K shared out.
int cut_linear(const z2z_ctx* c, SmallArgs& a) {
  a.tiles_n = a.N / S_T;
  return cut(a, rows_of_tiles(a.R) * a.tiles_n, 2 * c->num_cu, 4);
}
// A weight gradient, whose K is the rows, where those are many (forward and gradient, us: d = 256, d_ff = 704, 16000 rows 347 -> 169; d = d_ff = 64, 64000 rows 870 -> 61).
int cut_weight(const z2z_ctx* c, SmallArgs& a) { return cut(a, rows_of_tiles(a.R) * a.tiles_n, 4 * c->num_cu, 16); }

SmallArgs linear_args(const void* A, const void* W, bool k_major, const void* residual, void* out, bool f32, int R, const int32_t* rows_dev, int N, int K) {
  SmallArgs a = {};
  a.H = reinterpret_cast<const uint16_t*>(A);
  a.W = reinterpret_cast<const uint16_t*>(W);
  a.out = out;
  a.residual = residual;
  a.rows_dev = rows_dev;
  a.R = R;
  a.N = a.ldo = N;
  a.K = a.ldh = K;
  a.ldw = k_major ? N : K;
  a.f32 = f32 ? 1 : 0;
  return a;
}

SmallArgs weight_args(const z2z_small_weight& w, int rows, const int32_t* rows_dev) {
  SmallArgs a = {};
  a.H = reinterpret_cast<const uint16_t*>(w.A);
  a.W = reinterpret_cast<const uint16_t*>(w.W);
  a.out = w.out;
  a.residual = w.residual;
  a.k_dev = rows_dev;
  a.R = a.ldh = w.M;
  a.N = a.ldo = a.ldw = w.N;
  a.K = rows;
  a.tiles_n = w.N / S_T;
  return a;
}

}  // namespace

int z2z_launch_small_gated(const void* X, const void* W, int act, void* F, const z2z_ffn_kept& kept, int R, const int32_t* rows_dev, int d_ff, int K, hipStream_t s) {
  SmallArgs a = {};
  a.H = reinterpret_cast<const uint16_t*>(X);
  a.W = reinterpret_cast<const uint16_t*>(W);
  a.out = F;
  a.kept = kept;
  a.rows_dev = rows_dev;
  a.R = R;
  a.K = a.ldh = a.ldw = K;
  a.tiles_n = 2 * d_ff / S_T;
  a.d_ff = d_ff;
  a.act = act;
  return launch<false, 1, false>(a, 1, s);
}

int z2z_launch_small_slopes(z2z_ctx* c, const void* dY, const void* W, const z2z_ffn_kept& kept, void* slopes, int R, const int32_t* rows_dev, int d_ff, int K,
                            const z2z_small_weight* weight, hipStream_t s) {
  SmallArgs a = {};
  a.H = reinterpret_cast<const uint16_t*>(dY);
  a.W = reinterpret_cast<const uint16_t*>(W);
  a.out = slopes;
  a.kept = kept;
  a.rows_dev = rows_dev;
  a.R = R;
  a.K = a.ldh = K;
  a.ldw = a.d_ff = d_ff;
  a.ldo = 2 * d_ff;
  a.tiles_n = d_ff / S_T;
  if (!weight) return launch<true, 2, false>(a, 1, s);
  SmallArgs b = weight_args(*weight, R, rows_dev);
  const int parts = cut_weight(c, b);
  int rc = reserve(c, a, 1, &b, parts, s);
  if (rc == Z2Z_OK) rc = launch_pair<2, false>(a, 1, b, parts, s);
  return rc == Z2Z_OK ? add_up(b, parts, s) : rc;
}

int z2z_launch_small_linear(z2z_ctx* c, const void* A, const void* W, const void* residual, void* out, bool f32, int R, const int32_t* rows_dev, int N, int K,
                            hipStream_t s) {
  SmallArgs a = linear_args(A, W, false, residual, out, f32, R, rows_dev, N, K);
  const int parts = cut_linear(c, a);
  int rc = reserve(c, a, parts, nullptr, 1, s);
  if (rc == Z2Z_OK) rc = parts > 1 ? launch<false, 0, true>(a, parts, s) : launch<false, 0, false>(a, 1, s);
  return rc == Z2Z_OK ? add_up(a, parts, s) : rc;
}

int z2z_launch_small_parts(z2z_ctx* c, const void* A, const void* W, int R, const int32_t* rows_dev, int N, int K, const float** partial, int* ksplit,
                           hipStream_t s) {
  SmallArgs a = linear_args(A, W, false, nullptr, nullptr, false, R, rows_dev, N, K);
  const int parts = cut_linear(c, a);
  *ksplit = 0;
  if (parts <= 1) return Z2Z_OK;
  const int rc = reserve(c, a, parts, nullptr, 1, s);
  if (rc != Z2Z_OK) return rc;
  *partial = a.partial;
  *ksplit = parts;
  return launch<false, 0, true>(a, parts, s);
}

int z2z_launch_small_input(z2z_ctx* c, const void* A, const void* W, void* out, int R, const int32_t* rows_dev, int N, int K, const z2z_small_weight* weight,
                           hipStream_t s) {
  SmallArgs a = linear_args(A, W, true, nullptr, out, false, R, rows_dev, N, K), b = {};
  const int parts = cut_linear(c, a);
  int parts_b = 1;
  if (weight) {
    b = weight_args(*weight, R, rows_dev);
    parts_b = cut_weight(c, b);
  }
  int rc = reserve(c, a, parts, weight ? &b : nullptr, parts_b, s);
  if (rc != Z2Z_OK) return rc;
  if (weight)
    rc = parts > 1 ? launch_pair<0, true>(a, parts, b, parts_b, s) : launch_pair<0, false>(a, 1, b, parts_b, s);
  else
    rc = parts > 1 ? launch<true, 0, true>(a, parts, s) : launch<true, 0, false>(a, 1, s);
  if (rc == Z2Z_OK) rc = add_up(a, parts, s);
  return rc == Z2Z_OK ? add_up(b, parts_b, s) : rc;
}
