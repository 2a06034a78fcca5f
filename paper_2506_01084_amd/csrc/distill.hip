// Distillation over the extended vocabulary (gfx950): the loss of the joint softmax against a teacher's top logits, and its part of
// the gradient with respect to the logits.
//
// Section 2.4 of the zip2zip paper trains on the compressed sequence with one target code per position; here the target is a
// teacher's distribution q over K listed columns.  With p the joint softmax of section 2.3 at temperature T,
//   kl[r] = sum_k q_k (ln q_k - ln p_{id_k}),   ln p_v = logit[r, v] / T - lse[r],   q = softmax over the listed teacher logits / T.
// The log-sum-exp comes from the logits' kernels; only the K listed logits are needed besides.
#include "logits_common.h"

#include <algorithm>

namespace {

using namespace z2z_logits;

struct TeacherArgs {
  const int32_t* ids;       // [rows, K]
  const float* teacher;     // [rows, K]
  const int32_t* size;      // [sequences]
  int32_t rows, rows_per_seq, V, cap, K;
  float inv_t;
};

// A listed column this far below the best one (in logit / T) counts as nothing: e^-87 is next to the smallest normal number.
constexpr float kLeast = -87.f;
constexpr int T_GROUP = 8;

// A row's teacher in a wave: lane l has columns l + 64 u, u < PL (1 for lists of up to 64, else 4).  q = 0 where nothing is listed.
template <int PL>
struct Teacher {
  float q[PL], ln_q[PL];
  int32_t id[PL];           // -1: nothing listed
  bool some;                // the row has a distribution
  bool outside;             // some of it lies on a column that does not exist
};

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
  return x;
}

template <int PL>
__device__ __forceinline__ Teacher<PL> load_teacher(const TeacherArgs& a, int r, int columns) {
  const int lane = threadIdx.x & 63;
  Teacher<PL> t;
  float x[PL], m = kNegInf;
  bool nan = false;
#pragma unroll
  for (int u = 0; u < PL; ++u) {                     // (both on the way together)
    const size_t at = (size_t)r * a.K + min(lane + 64 * u, a.K - 1);
    t.id[u] = a.ids[at];
    x[u] = a.teacher[at];
  }
#pragma unroll
  for (int u = 0; u < PL; ++u) {
    if (lane + 64 * u >= a.K || t.id[u] < 0) {       // (what stands beside a column that is not listed counts for nothing)
      t.id[u] = -1;
      x[u] = kNegInf;
    }
    nan |= x[u] != x[u];
    m = fmaxf(m, x[u]);
  }
  m = wave_max(m);
  const bool any_nan = __ballot(nan) != 0ull;
  t.some = m > kNegInf || any_nan;
  float s = 0.f;
#pragma unroll
  for (int u = 0; u < PL; ++u) {
    // (differences of the logits first: exact where they matter; an infinite maximum makes NaN)
    t.ln_q[u] = t.some ? (x[u] - m) * a.inv_t : 0.f;
    t.q[u] = t.some && t.id[u] >= 0 && !(t.ln_q[u] < kLeast) ? expf(t.ln_q[u]) : 0.f;
    s += t.q[u];
  }
  s = wave_sum(s);
  const float ln_s = logf(s);
  bool outside = false;
#pragma unroll
  for (int u = 0; u < PL; ++u) {
    t.ln_q[u] -= ln_s;
    t.q[u] = t.id[u] >= 0 && t.some ? t.q[u] / s : 0.f;
    outside |= t.id[u] >= columns && t.q[u] > 0.f;
  }
  t.outside = __ballot(outside) != 0ull;
  return t;
}

template <bool BF16>
__device__ __forceinline__ float dot16(const uint4& x, const uint4& y, float acc) {
  const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (BF16) {
      acc = fmaf(__uint_as_float(xs[e] << 16), __uint_as_float(ys[e] << 16), acc);
      acc = fmaf(__uint_as_float(xs[e] & 0xFFFF0000u), __uint_as_float(ys[e] & 0xFFFF0000u), acc);
    } else {
      acc = fmaf(__uint_as_float(xs[e]), __uint_as_float(ys[e]), acc);
    }
  }
  return acc;
}

// One workgroup per hidden row: its first `gather` waves, up to eight, take the listed columns in turn, eight at a time against one read of the hidden
// row; the others, where there are some, merge the row's parts (fold) into its log-sum-exp meanwhile, as logits_combine_kernel does; then wave 0 has the loss.  Bound by the gather of K rows of W per hidden row (popular ones come out of the caches): 8192 rows
// of 64 columns, d = 4096, 4.3 GB: 307 us with four at a time, 286 with eight.
template <bool BF16, int PL>
__global__ void __launch_bounds__(768) teacher_loss_kernel(TeacherArgs a, const uint4* H, const uint4* W_base, const uint4* W_hyper, int d, int gather,
                                                           z2z_fold fold, float* lse, float* kl, float* student) {
  __shared__ float z_row[Z2Z_MAX_TEACHER];
  __shared__ Triple merged[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x, b = r / a.rows_per_seq;
  const int columns = a.V + min(max(a.size[b], 0), a.cap);
  const int n_chunks = d / (BF16 ? 8 : 4);
  const uint4* h = H + (size_t)r * n_chunks;
  constexpr int G = T_GROUP;
  const int mergers = (int)(blockDim.x >> 6) - gather;
  if (wave >= gather) {
    const size_t at = (size_t)r * fold.n_parts;
    const Triple tr = merge_parts(fold.m + at, fold.s + at, fold.i + at, (wave - gather) * 64 + lane, 64 * mergers, fold.n_parts, fold.inv_t);
    if (lane == 0) merged[wave - gather] = tr;
  }
  for (int k0 = wave < gather ? wave * G : a.K; k0 < a.K; k0 += gather * G) {
    const uint4* w[G];
    bool there[G];
    float acc[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int id = k0 + g < a.K ? a.ids[(size_t)r * a.K + k0 + g] : -1;
      there[g] = id >= 0 && id < columns;
      w[g] = !there[g] ? W_base : (id < a.V ? W_base + (size_t)id * n_chunks : W_hyper + ((size_t)b * a.cap + (id - a.V)) * n_chunks);
      acc[g] = 0.f;
    }
    for (int c = lane; c < n_chunks; c += 64) {
      const uint4 x = h[c];
      uint4 y[G];
#pragma unroll
      for (int g = 0; g < G; ++g) y[g] = w[g][c];
#pragma unroll
      for (int g = 0; g < G; ++g) acc[g] = dot16<BF16>(x, y[g], acc[g]);
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      acc[g] = wave_sum(acc[g]);
      if (lane == 0 && k0 + g < a.K) z_row[k0 + g] = there[g] ? acc[g] : 0.f;
    }
  }
  __syncthreads();
  for (int k = threadIdx.x; k < a.K; k += (int)blockDim.x) student[(size_t)r * a.K + k] = z_row[k];
  if (wave != 0) return;
  const Teacher<PL> t = load_teacher<PL>(a, r, columns);
  float l;
  if (mergers > 0) {
    Triple tr = merged[0];
    for (int w = 1; w < mergers; ++w) merge_triple(tr, merged[w], fold.inv_t);
    l = fmaf(tr.m, fold.inv_t, logf(tr.s));
    if (lane == 0) lse[r] = l;
  } else {
    l = lse[r];
  }
  float sum = 0.f;
#pragma unroll
  for (int u = 0; u < PL; ++u)
    if (t.q[u] != 0.f) sum += t.q[u] * (t.ln_q[u] - fmaf(z_row[min(lane + 64 * u, a.K - 1)], a.inv_t, -l));
  sum = wave_sum(sum);
  if (lane == 0) kl[r] = !t.some ? 0.f : (t.outside ? INFINITY : sum);
}

struct WeightArgs {
  const float *lse, *student, *grad;
  float *weight, *row_grad;
  int32_t* no_target;
  uint4* slot;              // 16-byte pieces of it
  size_t slot_pieces;
  int32_t row_blocks;
};

// The first row_blocks: dZ = g (p - q) of a row's listed columns, from the row's own logits, a wave per row; a column listed several times has the
// sum of its q, and its value at the first place.  g = the row's upstream gradient (1 without one) / T, 0 for rows without a distribution or with
// some of it on a column that does not exist; the probability epilogue stores g p everywhere and takes no target out.  The other blocks clear the slots.
template <int PL>
__global__ void __launch_bounds__(256) teacher_weight_kernel(TeacherArgs a, WeightArgs w) {
  if ((int)blockIdx.x >= w.row_blocks) {
    const size_t step = (size_t)(gridDim.x - (unsigned)w.row_blocks) * 256;
    for (size_t i = (size_t)(blockIdx.x - (unsigned)w.row_blocks) * 256 + threadIdx.x; i < w.slot_pieces; i += step) w.slot[i] = uint4{~0u, ~0u, ~0u, ~0u};
    return;
  }
  const int lane = threadIdx.x & 63;
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= a.rows) return;
  const int columns = a.V + min(max(a.size[r / a.rows_per_seq], 0), a.cap);
  const Teacher<PL> t = load_teacher<PL>(a, r, columns);
  const float gr = t.some && !t.outside ? (w.grad ? w.grad[r] : 1.0f) * a.inv_t : 0.f;
  if (lane == 0) {
    w.row_grad[r] = gr;
    w.no_target[r] = -1;
  }
  float total[PL];
  bool again[PL];
#pragma unroll
  for (int u = 0; u < PL; ++u) {
    total[u] = 0.f;
    again[u] = false;
  }
#pragma unroll
  for (int v = 0; v < PL; ++v) {
    if (64 * v >= a.K) break;
    const int n = min(64, a.K - 64 * v);
    for (int l = 0; l < n; ++l) {
      const int id = __builtin_amdgcn_readlane(t.id[v], l);
      const float q = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(t.q[v]), l));
#pragma unroll
      for (int u = 0; u < PL; ++u) {
        total[u] += id == t.id[u] ? q : 0.f;
        again[u] |= id == t.id[u] && 64 * v + l < 64 * u + lane;
      }
    }
  }
  const float l = w.lse[r];
#pragma unroll
  for (int u = 0; u < PL; ++u) {
    const int k = lane + 64 * u, id = t.id[u];
    if (k >= a.K) continue;
    const size_t at = (size_t)r * a.K + k;
    const bool there = id >= 0 && id < columns && gr != 0.f;
    w.weight[at] = there && !again[u] ? gr * (expf(fmaf(w.student[at], a.inv_t, -l)) - total[u]) : 0.f;
  }
}

// Zeros in the listed columns of dZ, behind the kernel that has stored g p everywhere: what stands there is the weights' part of the products.
__global__ void __launch_bounds__(256) teacher_dz_kernel(TeacherArgs a, uint16_t* base, size_t ld_base, uint16_t* hyper, size_t ld_hyper) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const int r = (int)(i / a.K);
  if (r >= a.rows) return;
  const int id = a.ids[i];
  if (id < 0) return;
  if (id < a.V)
    base[(size_t)r * ld_base + id] = 0;
  else if (id - a.V < min(max(a.size[r / a.rows_per_seq], 0), a.cap))
    hyper[(size_t)r * ld_hyper + (id - a.V)] = 0;
}

TeacherArgs teacher_args(const z2z_ctx* c, const z2z_teacher& t, int r0, int rows, int rows_per_seq) {
  TeacherArgs a;
  a.ids = t.ids + (size_t)r0 * t.K;
  a.teacher = t.logits + (size_t)r0 * t.K;
  a.size = c->st.size + r0 / rows_per_seq;
  a.rows = rows;
  a.rows_per_seq = rows_per_seq;
  a.V = c->cfg.V;
  a.cap = c->cfg.cap;
  a.K = t.K;
  a.inv_t = 1.0f / t.temperature;
  return a;
}

}  // namespace

int z2z_launch_extended_distill(z2z_ctx* c, const void* H, int32_t rows, int32_t rows_per_seq, const void* W_base, const void* W_hyper,
                                const z2z_teacher& t, float* kl, float* lse, float* student, hipStream_t s) {
  // The parts' merge in the loss's launch, a launch less, in waves of its own: with up to 40 columns, whose workgroups are small enough to have a CU's
  // wave slots left, and with more for up to 512 rows.  Apart / together, us, T = 2: fp32 V = 5000, d = 128, 122 rows, 33 columns 21.1 / 17.8, V = 32000, d = 256
  // 36.4 / 32.8, 351 rows 73.6 / 69.8; bf16 V = 50257, d = 1024, 122 rows 35.8 / 32.2, 4096 454 / 451, of 64 columns 351 rows 76.4 / 76.0, 1000 144 /
  // 147, 4096 486 / 508.
  const int gather = std::min((t.K + T_GROUP - 1) / T_GROUP, 8);
  const bool together = gather <= 5 || rows <= 512;
  if ((long long)rows * 64 * (gather + 4) > kLaunchThreads) return Z2Z_EUNSUPPORTED;
  z2z_fold fold = {};
  const int rc = z2z_launch_extended_logits(c, H, rows, rows_per_seq, W_base, W_hyper, nullptr, nullptr, lse, nullptr, s, false, t.temperature,
                                            together ? &fold : nullptr);
  if (rc != Z2Z_OK) return rc;
  const TeacherArgs a = teacher_args(c, t, 0, rows, rows_per_seq);
  const uint4 *h = reinterpret_cast<const uint4*>(H), *wb = reinterpret_cast<const uint4*>(W_base), *wh = reinterpret_cast<const uint4*>(W_hyper);
  const dim3 grid((unsigned)rows), block(64u * (unsigned)(gather + (fold.n_parts > 256 ? 4 : fold.n_parts > 0 ? 1 : 0)));
  if (c->cfg.dtype == Z2Z_BF16 && t.K <= 64)
    hipLaunchKernelGGL((teacher_loss_kernel<true, 1>), grid, block, 0, s, a, h, wb, wh, c->cfg.d, gather, fold, lse, kl, student);
  else if (c->cfg.dtype == Z2Z_BF16)
    hipLaunchKernelGGL((teacher_loss_kernel<true, 4>), grid, block, 0, s, a, h, wb, wh, c->cfg.d, gather, fold, lse, kl, student);
  else if (t.K <= 64)
    hipLaunchKernelGGL((teacher_loss_kernel<false, 1>), grid, block, 0, s, a, h, wb, wh, c->cfg.d, gather, fold, lse, kl, student);
  else
    hipLaunchKernelGGL((teacher_loss_kernel<false, 4>), grid, block, 0, s, a, h, wb, wh, c->cfg.d, gather, fold, lse, kl, student);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

int z2z_launch_teacher_weight(z2z_ctx* c, const z2z_teacher& t, int rows, int rows_per_seq, const float* lse, const float* grad,
                              const z2z_listed_part& l, hipStream_t s) {
  const TeacherArgs a = teacher_args(c, t, 0, rows, rows_per_seq);
  const size_t keys = (size_t)c->cfg.V + (size_t)c->cfg.B * c->cfg.cap;
  WeightArgs w;
  w.lse = lse;
  w.student = t.student;
  w.grad = grad;
  w.weight = l.weight;
  w.row_grad = l.row_grad;
  w.no_target = l.no_target;
  w.slot = reinterpret_cast<uint4*>(l.slot);
  w.slot_pieces = (keys + 3) / 4;                    // (its room is a multiple of 256 bytes)
  w.row_blocks = (rows + 3) / 4;
  const dim3 grid((unsigned)w.row_blocks + (unsigned)std::min<size_t>((w.slot_pieces + 255) / 256, 1024)), block(256);
  if (t.K <= 64)
    hipLaunchKernelGGL(teacher_weight_kernel<1>, grid, block, 0, s, a, w);
  else
    hipLaunchKernelGGL(teacher_weight_kernel<4>, grid, block, 0, s, a, w);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

int z2z_launch_teacher_dz(z2z_ctx* c, const z2z_teacher& t, int r0, int rows, int rows_per_seq, void* base, size_t ld_base, void* hyper,
                          size_t ld_hyper, hipStream_t s) {
  const TeacherArgs a = teacher_args(c, t, r0, rows, rows_per_seq);
  hipLaunchKernelGGL(teacher_dz_kernel, dim3((unsigned)(((long long)rows * t.K + 255) / 256)), dim3(256), 0, s, a, reinterpret_cast<uint16_t*>(base),
                     ld_base, reinterpret_cast<uint16_t*>(hyper), ld_hyper);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}
