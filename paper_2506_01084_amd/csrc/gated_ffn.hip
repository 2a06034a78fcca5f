// The gated feed-forward block of a learned hyper-encoder's layer, forward and backward (zip2zip paper, section 2.2; the paper names a transformer and no
// more of its block): Y = (act(X W1[:f]^T) * (X W1[f:]^T)) W2^T + residual.
//
// Forward, many rows: one launch of the tile kernel for both projections, activation and product (a tile of 256 weight rows is 128 gate columns and the same 128
// of the other projection), one for the product with W2; fewer take smaller tiles (small_tile.hip).  Few rows are bound by the weights' bytes: the weight-streaming kernel, in bf16 or from 4 bits (q4.hip), leaves
// parts of the products, whose sum applies the activation.  Backward: dF = dY W2 becomes dG | dU in the epilogue; then dW2 = dY^T F,
// dW1 = [dG | dU]^T X, dX = [dG | dU] W1, all on operands as they are.
#include "few_rows.h"
#include "gated.h"
#include "small_tile.h"

#include <algorithm>

namespace {

// More rows than this, and 4-bit weights are expanded to bf16 first: the products are the matrix cores' work then.  (us, 300 rows from 4 bits / 330 expanded: d = 4096, d_ff = 10944
// 155 / 245; 3584, 9600 115 / 204; 2048, 5504 62 / 79; 1024, 2752 31 / 38; 400 rows expanded 244, 202, 81, 38.)
constexpr int kExpandRows = 320;

__global__ void __launch_bounds__(256) fill_zero_kernel(uint4* p, size_t n, uint4* q, size_t n_q) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n + n_q; i += (size_t)gridDim.x * 256) {
    uint4* at = i < n ? p + i : q + (i - n);
    *at = uint4{0u, 0u, 0u, 0u};
  }
}

// F and its factors out of pairs of 16 bits: the matrices that the gradient's products and their epilogues read.  Bound by memory, 12 bytes an element.
__global__ void __launch_bounds__(256) kept_pairs_kernel(const uint4* pairs, size_t quads, int act, z2z_ffn_kept to) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < quads; i += (size_t)gridDim.x * 256) {
    const uint4 v = pairs[i];
    const float g[4] = {z2z_gated::of_code16(v.x), z2z_gated::of_code16(v.y), z2z_gated::of_code16(v.z), z2z_gated::of_code16(v.w)};
    const float u[4] = {z2z_gated::of_code16(v.x >> 16), z2z_gated::of_code16(v.y >> 16), z2z_gated::of_code16(v.z >> 16), z2z_gated::of_code16(v.w >> 16)};
    reinterpret_cast<uint2*>(to.f)[i] = z2z_gated::hidden_and_keep4(g, u, act, to, 4 * i);
  }
}

// Rows up to which the products run on the kernel that shares nothing between workgroups but has no parts to add up (few_rows.hip): every workgroup reads all rows, which
// costs more than the others' sums, or tiles, from a number on that depends on the weights.  us, that kernel / the others:
//   bf16   d = 4096, d_ff = 10944  1 row 47 / 54, 16 rows 57 / 61, 24 70 / 65;   2048, 5504  1 19.8 / 23.7, 16 25.7 / 24.7, 24 31.1 / 27.4;   1024, 2752  1 10.5 / 14.5, 16 12.2 / 15.2,
//          33 17.4 / 15.8;   512, 1408  33 11.5 / 13.1, 65 14.4 / 13.4;   256, 704  237 10.3 / 12.9
//   4 bits d = 4096, d_ff = 10944, group 64  1 19.8 / 26.6, 4 21.7 / 27.8, 16 32.2 / 29.6;   3584, 9600, 128  4 17.8 / 21.6, 16 27.2 / 24.6;   2048, 5504, 32  4 13.7 / 15.1, 16 18.0 / 18.3,
//          32 26.8 / 24.5;   1024, 2752, 64  1 8.3 / 13.1, 32 12.8 / 15.5, 64 20.1 / 20.6, 128 24.5 / 26.5
bool few_rows(const z2z_ffn* f, int d, int R) {
  if (f->group) return R <= 8 || ((long long)d * f->d_ff <= (1 << 22) && R <= 64);
  return R <= 16 || (R <= 256 && (long long)R * d * f->d_ff <= (3 << 24));
}

// Rows times d times d_ff up to which a product runs on tiles of 64 x 64 (small_tile.hip): more, and its 256 x 256 tiles keep enough CUs busy.  us of a product, or of
// the two of a forward pass, with the others / on small tiles:
//   forward    d = 1024, d_ff = 2752  65 rows 25.6 / 18.0, 300 53 / 24, 2000 93 / 62, 4000 114 / 151;   2048, 5504  100 39.7 / 30.2, 500 80 / 67, 700 94 / 93, 1000 99 / 113;   3584, 9600  65 62.4 / 59.5,
//              160 92 / 76, 300 121 / 136;   4096, 10944  65 of weights that no cache holds: 78 / 86
//   dF         1024, 2752  2000 -13 us, 4000 +10;   2048, 5504  1000 -5, 1500 +7;   3584, 9600  237 -3, 500 +9
//   dX         1024, 2752  1000 -8, 1500 +1;   2048, 5504  237 -12, 500 +1;   4096, 10944  16 -11, 65 -3, 100 0: alone
//   all three, two in a launch (forward and gradient)   1024, 2752  237 122 / 57, 1500 248 / 172, 2000 276 / 234;   2048, 5504  16 83 / 69, 237 129 / 124, 500 200 / 201;   3584, 9600
//              65 230 / 211, 128 249 / 254;   4096, 10944  16 225 / 202, 33 231 / 232, 100 286 / 308;   512, 1408  4000 214 / 155, 8000 257 / 286;   256, 704  20000 271 / 207, 30000 347 / 315
constexpr long long kSmallForward = 3ll << 31, kSmallSlopes = 5ll << 31, kSmallInput = 3ll << 30, kSmallGradient = 5ll << 30;

bool small_tiles(const z2z_ffn* f, int d, int R, long long most) { return (long long)d * f->d_ff * R <= most; }
// (Weights that the memory-side cache does not hold are read for every 64 rows.)
bool held(const z2z_ffn* f, int d) { return (size_t)3 * d * f->d_ff * sizeof(uint16_t) <= 2 * z2z_logits::kKeepBytes; }
bool small_forward(const z2z_ffn* f, int d, int R) { return small_tiles(f, d, R, kSmallForward) && held(f, d); }
bool small_gradient(const z2z_ffn* f, int d, int R) { return small_tiles(f, d, R, kSmallGradient) && (R <= 16 || held(f, d)); }

size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

}  // namespace

size_t z2z_ffn_work(const z2z_ffn* f, int d, int rows) {
  return padded((size_t)rows * f->d_ff * 2) + (f->group && rows > kExpandRows ? (size_t)3 * d * f->d_ff * 2 : 0);
}

int z2z_launch_ffn_hidden(z2z_ctx* c, const void* X, const z2z_ffn* f, const z2z_ffn_kept& kept, int R, const int32_t* rows_dev, void* work, z2z_ffn_out* out,
                          hipStream_t s) {
  const int d = c->cfg.d, dff = f->d_ff;
  unsigned char* F = kept.f ? reinterpret_cast<unsigned char*>(kept.f) : reinterpret_cast<unsigned char*>(work);
  const void* w1 = f->w_1;
  *out = z2z_ffn_out{F, f->w_2, nullptr, 0, dff, false, false, false};
  if (few_rows(f, d, R)) {
    out->scale = f->scale_2;
    out->group = f->group;
    out->few = true;
    return z2z_launch_few_gated(X, w1, f->scale_1, f->group, f->act, F, kept, R, rows_dev, dff, d, s);
  }
  if (f->group && R <= kExpandRows) {
    out->scale = f->scale_2;
    out->group = f->group;
    const float* partial = nullptr;
    int ksplit = 0;
    const int rc = z2z_launch_q4_parts(c, X, w1, f->scale_1, f->group, R, rows_dev, 2 * dff, d, &partial, &ksplit, s);
    if (rc != Z2Z_OK) return rc;
    return z2z_launch_gated_sum(partial, ksplit, R, rows_dev, dff, f->act, F, z2z_ffn_kept{}, s);
  }
  if (f->group) {
    unsigned char *e1 = F + padded((size_t)R * dff * 2), *e2 = e1 + (size_t)2 * dff * d * 2;
    int rc = z2z_launch_expand_q4(w1, f->scale_1, 2 * dff, d, f->group, e1, s);
    if (rc != Z2Z_OK) return rc;
    rc = z2z_launch_expand_q4(f->w_2, f->scale_2, d, dff, f->group, e2, s);
    if (rc != Z2Z_OK) return rc;
    w1 = e1;
    out->w = e2;
  }
  if (small_forward(f, d, R)) {
    out->small = true;
    return z2z_launch_small_gated(X, w1, f->act, F, kept, R, rows_dev, dff, d, s);
  }
  // (few rows: does anything of the weights stay in the memory-side cache until the next call?)
  out->once = (size_t)3 * d * dff * sizeof(uint16_t) > z2z_logits::kKeepBytes;
  return z2z_launch_gated_hidden(c, X, w1, f->act, F, kept, R, rows_dev, dff, d, s, out->once);
}

int z2z_launch_ffn(z2z_ctx* c, const void* X, const z2z_ffn* f, const void* residual, void* Y, bool stream_f32, void* kept, int R, const int32_t* rows_dev,
                   void* work, hipStream_t s) {
  const int d = c->cfg.d;
  z2z_ffn_out o;
  int rc = z2z_launch_ffn_hidden(c, X, f, z2z_kept_in(kept, (size_t)R, f->d_ff, f->kept), R, rows_dev, work, &o, s);
  if (rc != Z2Z_OK) return rc;
  if (o.few) return z2z_launch_few_linear(o.F, o.w, o.scale, o.group, residual, Y, stream_f32, R, rows_dev, d, o.d_ff, s);
  if (o.small) return z2z_launch_small_linear(c, o.F, o.w, residual, Y, stream_f32, R, rows_dev, d, o.d_ff, s);
  if (!o.group) return z2z_launch_linear(c, o.F, o.w, nullptr, residual, 0, Y, R, rows_dev, d, o.d_ff, s, stream_f32, nullptr, o.once);
  const float* partial = nullptr;
  int ksplit = 0;
  rc = z2z_launch_q4_parts(c, o.F, o.w, o.scale, o.group, R, rows_dev, d, o.d_ff, &partial, &ksplit, s);
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_linear_sum(partial, ksplit, R, rows_dev, d, residual, Y, stream_f32, s);
}

size_t z2z_ffn_backward_work(const z2z_ffn* f, int rows) { return (size_t)rows * f->d_ff * (f->kept == Z2Z_KEPT_16 ? 4 + 8 : 4); }

int z2z_launch_ffn_backward(z2z_ctx* c, const void* X, const z2z_ffn* f, const void* kept, const void* dY, void* dX, const z2z_ffn* grad, bool add, int R,
                            const int32_t* rows_dev, void* work, hipStream_t s) {
  const int d = c->cfg.d, dff = f->d_ff;
  z2z_ffn_kept k = z2z_kept_in(const_cast<void*>(kept), (size_t)R, dff, f->kept);
  if (f->kept == Z2Z_KEPT_16) {
    const size_t quads = (size_t)R * dff / 4;
    k = z2z_kept_in(reinterpret_cast<unsigned char*>(work) + (size_t)R * dff * 4, (size_t)R, dff);
    hipLaunchKernelGGL(kept_pairs_kernel, dim3((unsigned)std::min<size_t>((quads + 255) / 256, 16384)), dim3(256), 0, s, reinterpret_cast<const uint4*>(kept), quads,
                       f->act, k);
  }
  void *dw1 = const_cast<void*>(grad->w_1), *dw2 = const_cast<void*>(grad->w_2);
  // on small tiles the weight gradients go along with the products beside them
  const bool weights = small_gradient(f, d, R), input = weights || small_tiles(f, d, R, kSmallInput);
  const z2z_small_weight w1 = {work, X, add ? dw1 : nullptr, dw1, 2 * dff, d}, w2 = {dY, k.f, add ? dw2 : nullptr, dw2, d, dff};
  int rc = small_tiles(f, d, R, kSmallSlopes) ? z2z_launch_small_slopes(c, dY, f->w_2, k, work, R, rows_dev, dff, d, weights ? &w2 : nullptr, s)
                                              : z2z_launch_gated_slopes(c, dY, f->w_2, k, work, R, rows_dev, dff, d, s);
  if (rc == Z2Z_OK && !weights) {
    rc = z2z_launch_linear_weight(c, dY, d, k.f, dff, R, rows_dev, add ? dw2 : nullptr, dw2, d, dff, s);
    if (rc == Z2Z_OK) rc = z2z_launch_linear_weight(c, work, 2 * dff, X, d, R, rows_dev, add ? dw1 : nullptr, dw1, 2 * dff, d, s);
  }
  if (rc != Z2Z_OK) return rc;
  if (input) return z2z_launch_small_input(c, work, f->w_1, dX, R, rows_dev, d, 2 * dff, weights ? &w1 : nullptr, s);
  return z2z_launch_linear_input(c, work, 2 * dff, f->w_1, d, 2 * dff, nullptr, dX, d, R, rows_dev, d, 2 * dff, s, {1, 0, 0}, 0, kGatedMinSaved);
}

int z2z_launch_fill_zero(void* p, size_t bytes, void* q, size_t bytes_q, hipStream_t s) {
  hipLaunchKernelGGL(fill_zero_kernel, dim3(1024), dim3(256), 0, s, reinterpret_cast<uint4*>(p), bytes / 16, reinterpret_cast<uint4*>(q), bytes_q / 16);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}
