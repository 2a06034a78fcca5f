// The gated feed-forward block of a learned hyper-encoder's layer, forward and backward (zip2zip paper, section 2.2; the paper names a transformer and no
// more of its block): Y = (act(X W1[:f]^T) * (X W1[f:]^T)) W2^T + residual.
//
// Forward, many rows: one launch of the tile kernel for both projections, activation and product (a tile of 256 weight rows is 128 gate columns and the same 128
// of the other projection), one for the product with W2.  Few rows are bound by the weights' bytes: the weight-streaming kernel, in bf16 or from 4 bits (q4.hip), leaves
// parts of the products, whose sum applies the activation.  Backward: dF = dY W2 becomes dG | dU and F in the epilogue; then dW2 = dY^T F,
// dW1 = [dG | dU]^T X, dX = [dG | dU] W1, all on operands as they are.
#include "logits_common.h"

namespace {

// Rows from which on 4-bit weights are expanded to bf16 first: the products are the matrix cores' work then.
constexpr int kExpandRows = 192;

__global__ void __launch_bounds__(256) fill_zero_kernel(uint4* p, size_t n, uint4* q, size_t n_q) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n + n_q; i += (size_t)gridDim.x * 256) {
    uint4* at = i < n ? p + i : q + (i - n);
    *at = uint4{0u, 0u, 0u, 0u};
  }
}

size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

}  // namespace

size_t z2z_ffn_work(const z2z_ffn* f, int d, int rows) {
  return padded((size_t)rows * f->d_ff * 2) + (f->group && rows > kExpandRows ? (size_t)3 * d * f->d_ff * 2 : 0);
}

int z2z_launch_ffn_hidden(z2z_ctx* c, const void* X, const z2z_ffn* f, void* kept, int R, const int32_t* rows_dev, void* work, z2z_ffn_out* out,
                          hipStream_t s) {
  const int d = c->cfg.d, dff = f->d_ff;
  unsigned char* F = reinterpret_cast<unsigned char*>(work);
  const void* w1 = f->w_1;
  *out = z2z_ffn_out{F, f->w_2, nullptr, 0, dff, false};
  if (f->group && R <= kExpandRows) {
    out->scale = f->scale_2;
    out->group = f->group;
    const float* partial = nullptr;
    int ksplit = 0;
    const int rc = z2z_launch_q4_parts(c, X, w1, f->scale_1, f->group, R, rows_dev, 2 * dff, d, &partial, &ksplit, s);
    if (rc != Z2Z_OK) return rc;
    return z2z_launch_gated_sum(partial, ksplit, R, rows_dev, dff, f->act, F, nullptr, s);
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
  // (few rows: does anything of the weights stay in the memory-side cache until the next call?)
  out->once = (size_t)3 * d * dff * sizeof(uint16_t) > z2z_logits::kKeepBytes;
  return z2z_launch_gated_hidden(c, X, w1, f->act, F, kept, R, rows_dev, dff, d, s, out->once);
}

int z2z_launch_ffn(z2z_ctx* c, const void* X, const z2z_ffn* f, const void* residual, void* Y, bool stream_f32, void* kept, int R, const int32_t* rows_dev,
                   void* work, hipStream_t s) {
  const int d = c->cfg.d;
  z2z_ffn_out o;
  int rc = z2z_launch_ffn_hidden(c, X, f, kept, R, rows_dev, work, &o, s);
  if (rc != Z2Z_OK) return rc;
  if (!o.group) return z2z_launch_linear(c, o.F, o.w, nullptr, residual, 0, Y, R, rows_dev, d, o.d_ff, s, stream_f32, nullptr, o.once);
  const float* partial = nullptr;
  int ksplit = 0;
  rc = z2z_launch_q4_parts(c, o.F, o.w, o.scale, o.group, R, rows_dev, d, o.d_ff, &partial, &ksplit, s);
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_linear_sum(partial, ksplit, R, rows_dev, d, residual, Y, stream_f32, s);
}

size_t z2z_ffn_backward_work(const z2z_ffn* f, int rows) { return padded((size_t)rows * f->d_ff * 2) + (size_t)rows * 2 * f->d_ff * 2; }

int z2z_launch_ffn_backward(z2z_ctx* c, const void* X, const z2z_ffn* f, const void* kept, const void* dY, void* dX, const z2z_ffn* grad, bool add, int R,
                            const int32_t* rows_dev, void* work, hipStream_t s) {
  const int d = c->cfg.d, dff = f->d_ff;
  unsigned char *F = reinterpret_cast<unsigned char*>(work), *slopes = F + padded((size_t)R * dff * 2);
  void *dw1 = const_cast<void*>(grad->w_1), *dw2 = const_cast<void*>(grad->w_2);
  int rc = z2z_launch_gated_slopes(c, dY, f->w_2, kept, f->act, slopes, F, R, rows_dev, dff, d, s);
  if (rc != Z2Z_OK) return rc;
  rc = z2z_launch_linear_weight(c, dY, d, F, dff, R, rows_dev, add ? dw2 : nullptr, dw2, d, dff, s);
  if (rc != Z2Z_OK) return rc;
  rc = z2z_launch_linear_weight(c, slopes, 2 * dff, X, d, R, rows_dev, add ? dw1 : nullptr, dw1, 2 * dff, d, s);
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_linear_input(c, slopes, 2 * dff, f->w_1, d, 2 * dff, nullptr, dX, d, R, rows_dev, d, 2 * dff, s);
}

int z2z_launch_fill_zero(void* p, size_t bytes, void* q, size_t bytes_q, hipStream_t s) {
  hipLaunchKernelGGL(fill_zero_kernel, dim3(1024), dim3(256), 0, s, reinterpret_cast<uint4*>(p), bytes / 16, reinterpret_cast<uint4*>(q), bytes_q / 16);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}
