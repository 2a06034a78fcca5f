// Internal declarations shared by the translation units of libz2z (HIP, gfx950 only).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "z2z.h"

#define Z2Z_API __attribute__((visibility("default")))
#define Z2Z_MAX_TIMED 1024

// Per-sequence codebook storage, all in device global memory and owned by the context.
//   size[b]                    number of entries C_b
//   prev_code[b], prev_len[b]  last phrase emitted / consumed (-1, 0 = none)
//   ent_tokens[b][e][0..M)     flattened base tokens of entry e, -1 padded
//   ent_len[b][e]              its length (0 = unused)
//   slots[b][h]                open-addressing hash table over the trie edges, one 64-bit word per slot:
//                              parent code (24 bits) | last token (24 bits) | entry index (16 bits); all
//                              ones = empty.  Hence V + cap <= 2^24.
struct LzwState {
  int32_t* size;
  int32_t* prev_code;
  int32_t* prev_len;
  int32_t* rounds;           // [B] rounds the latest parse kernel took for the sequence (instrumentation)
  int32_t* tail;             // [B, 3] codes and tokens up to where the latest decode call left the window kernel, codes in all
  int32_t* ent_tokens;
  int32_t* ent_len;
  unsigned long long* slots;
  int32_t V, M, cap, nslots;
  int32_t slots_fit_lds;     // the table of one sequence fits the LDS of a CU
  int32_t tags_fit_lds;      // it does not, but a tag of every slot does
};

// Where the tile kernels leave their partial (max, sum-exp, argmax) triples: three arrays of `capacity`
// elements each.  Either the context's growable buffers or a device's static array.
struct z2z_parts {
  float* m;
  float* s;
  int32_t* i;
  size_t capacity;
};

// The parts that a logits call has left, [rows, n_parts], and the 1 / T of their sums.
struct z2z_fold {
  const float *m, *s;
  const int32_t* i;
  int32_t n_parts;
  float inv_t;
};

// A work buffer of the context that grows with the calls.
struct z2z_work {
  void* p;
  size_t bytes;
  bool named;              // a call that uses it has been captured into a graph
};

// Memory of work buffers that had to grow although a graph names it.
struct z2z_kept {
  void* p;
  z2z_kept* next;
};

struct z2z_ctx {
  z2z_config cfg;
  int device;
  int lds_limit;           // bytes of LDS one workgroup may use on this device
  int num_cu;
  LzwState st;
  float coef[Z2Z_MAX_M + 1][Z2Z_MAX_M];   // coef[L][j]: pooling coefficient of token j of a length-L entry
  // extended_logits scratch: partial (max, sum-exp, argmax) per (part, row), in parts_ws
  z2z_work parts_ws;
  float* part_m;
  float* part_s;
  int32_t* part_i;
  size_t part_capacity;    // elements in each of the three arrays
  // extended_sample scratch: best perturbed value and the scaled logit at that column (its column is part_i), in draws_ws
  z2z_work draws_ws;
  float* part_v;
  float* part_l;
  // truncated sampling: the rows' logits as the decode kernel stores them, and the row maxima, in sample_ws
  z2z_work sample_ws;
  float* sample_logits;
  float* row_max;
  int trunc_ready;
  // hyper_encode work space: the activations of one pass (bf16)
  z2z_work enc_ws;
  size_t enc_ws_refused;   // 0, or a size the device had no room for
  z2z_work enc_bwd_ws;     // saved activations and gradients of the learned encoder's backward pass
  bool enc_kept;           // the work space holds the rows of a z2z_hyper_encode_keep call ...
  size_t enc_kept_need;    // ... laid out for this size ...
  const void* enc_kept_E;  // ... computed from this embedding matrix
  z2z_work bwd_ws;         // backward pass of the loss: dZ of both parts (bf16), the row gradients
  void* prune_prefix;      // codebook pruning: every entry's prefix entry (scratch, [B, cap] int32)
  void* coef_dev;          // the pooling coefficients on the device (pooling backward)
  // dense layers on few rows with K split over workgroups: the partial tiles
  z2z_work partial_ws;
  z2z_work lookup_ws;      // gradient of the code lookup: sorted positions, sums that cross pieces; a teacher's listed part
  z2z_work ffn_ws;         // gated feed-forward block: hidden layer, its gradients, weights expanded from 4 bits
  z2z_work clip_ws;        // sums of the gradients' squares
  bool capturing;          // the present call is being captured into a graph, or may be
  z2z_kept* kept;
  // options
  int opt_backward_chunk;
  int opt_logits_kernel, opt_logits_strip, opt_lzw_kernel, opt_decode_kernel, opt_timing, opt_logits_map,
      opt_sample_kernel;
  int decode_ready;        // the decode-step logits kernel can be launched for this configuration
  int skinny_ready;        // the decode-step kernel's LDS fits this device (dense layers on few rows use it)
  int fast_ready;          // the 128 KiB-LDS bf16 logits kernel can be launched on this device
  int mid_ready;           // the weight-streaming kernel for up to 192 hidden rows can be launched on this device
  // timing record
  hipEvent_t ev_start[Z2Z_MAX_TIMED];
  hipEvent_t ev_stop[Z2Z_MAX_TIMED];
  int n_timed;
  int ev_created;
  long long n_launch[Z2Z_N_KERNEL_FAMILIES];   // launches enqueued per logits kernel family
};

// What a row is distilled from (z2z_extended_distill).
struct z2z_teacher {
  int32_t K;
  const int32_t* ids;      // [rows, K]
  const float* logits;     // [rows, K]
  float temperature;
  const float* student;    // [rows, K] the student's logits there (backward)
};

// launchers (each validates nothing: the C-ABI layer has done so)
int z2z_lzw_prepare(z2z_ctx* c);   // raises the dynamic-LDS ceiling of the parse kernels
int z2z_launch_lzw_reset(z2z_ctx* c, hipStream_t s);
int z2z_launch_lzw_encode(z2z_ctx* c, const int32_t* tokens, const int32_t* lens, int32_t stride, int32_t flags,
                          int32_t* codes, int32_t* n_codes, int32_t out_stride, int32_t* status, hipStream_t s);
int z2z_launch_lzw_decode(z2z_ctx* c, const int32_t* codes, const int32_t* n_codes, int32_t stride, int32_t flags,
                          int32_t* tokens, int32_t* n_tokens, int32_t out_stride, int32_t* status, hipStream_t s);
int z2z_launch_step_update(z2z_ctx* c, const int32_t* codes, int32_t stride, const void* E, void* W_hyper,
                           int32_t* n_tokens, int32_t* status, hipStream_t s);
int z2z_launch_codebook_usage(z2z_ctx* c, const int32_t* codes, const int32_t* n_codes, int32_t stride, int32_t* usage,
                              hipStream_t s);
int z2z_launch_codebook_prune(z2z_ctx* c, const int32_t* keep, int32_t* new_id, int32_t* n_kept, hipStream_t s);
int z2z_launch_codebook_prefill(z2z_ctx* c, const int32_t* phrases, const int32_t* phrase_len, const int32_t* counts,
                                int32_t n_max, int32_t flags, int32_t* n_added, int32_t* status, hipStream_t s);
int z2z_launch_hyper_embed(z2z_ctx* c, const void* E, void* W_hyper, const int32_t* first, int32_t max_new,
                           hipStream_t s);
// use_static: the partial triples go to the device's static array (nothing is allocated; Z2Z_ELIMIT when they
// do not fit) instead of the context's growable buffers
int z2z_launch_extended_logits(z2z_ctx* c, const void* H, int32_t rows, int32_t rows_per_seq, const void* W_base,
                               const void* W_hyper, int32_t* argmax, float* mx, float* lse, float* logits,
                               hipStream_t s, bool use_static = false, float temperature = 1.0f, z2z_fold* fold = nullptr);   // fold: the parts are left to the caller
int z2z_static_scratch_prepare(z2z_ctx* c);   // z2z_create: look up the static array's address on c->device
int z2z_launch_extended_sample(z2z_ctx* c, const void* H, int32_t rows, int32_t rows_per_seq, const void* W_base,
                               const void* W_hyper, float temperature, int32_t top_k, float top_p, uint64_t seed,
                               uint64_t step, int32_t* token, float* logprob, hipStream_t s);
int z2z_sample_truncated_prepare(z2z_ctx* c);
int z2z_launch_extended_nll_backward(z2z_ctx* c, const void* H, int32_t rows, int32_t rows_per_seq, const void* W_base,
                                     const void* W_hyper, const int32_t* targets, const float* lse,
                                     const float* grad_nll, void* dH, void* dW_base, void* dW_hyper, hipStream_t s,
                                     const z2z_teacher* teacher = nullptr);
int z2z_launch_hyper_embed_backward(z2z_ctx* c, const void* dW_hyper, float* dE, hipStream_t s);
bool z2z_hyper_encode_ok(const z2z_ctx* c, const z2z_encoder* enc);
int z2z_launch_hyper_encode(z2z_ctx* c, const void* E, const z2z_encoder* enc, void* W_hyper, const int32_t* first,
                            int32_t max_new, hipStream_t s);
int z2z_launch_hyper_encode_train(z2z_ctx* c, int mode, const void* E, const z2z_encoder* enc, void* W_hyper,
                                  const void* dW_hyper, const z2z_encoder* grad, float* dE, hipStream_t s);
int z2z_launch_extended_nll(z2z_ctx* c, const void* H, int32_t rows, int32_t rows_per_seq, const void* W_base,
                            const void* W_hyper, const int32_t* targets, float* nll, float* lse, hipStream_t s);

int z2z_launch_embed_codes(z2z_ctx* c, const int32_t* codes, const int32_t* n_codes, int32_t stride, const void* E, const void* W_hyper,
                           float scale, void* X, int32_t* status, hipStream_t s);
int z2z_launch_embed_codes_backward(z2z_ctx* c, const int32_t* codes, const int32_t* n_codes, int32_t stride, float scale, const void* dX,
                                    int32_t flags, float* dE, void* dW_hyper, hipStream_t s);
int z2z_launch_extended_distill(z2z_ctx* c, const void* H, int32_t rows, int32_t rows_per_seq, const void* W_base, const void* W_hyper,
                                const z2z_teacher& t, float* kl, float* lse, float* student, hipStream_t s);
// The backward pass's listed columns, for all rows of the call: dZ there (weight), and what it adds to the gradients, in fp32.
struct z2z_listed_part {
  float* weight;           // [rows, K]
  float* row_grad;         // [rows] of the probability epilogue
  int32_t* no_target;      // [rows] its targets: none
  float* hidden;           // [rows, d]: sum_k weight[r, k] W[ids[r, k]]
  int32_t* slot;           // [V + B * cap] where in sums a row of [W_base ; W_hyper[b]] has its sum of weight[r, k] H[r], -1: none lists it
  float* sums;             // rows of d
};
int z2z_listed_reserve(z2z_ctx* c, long long rows, int per_row, z2z_listed_part* l, hipStream_t s);
// weight, row_grad, no_target, and no slots yet; then hidden, slot and sums, the latter sorted by row (embed_codes.hip)
int z2z_launch_teacher_weight(z2z_ctx* c, const z2z_teacher& t, int rows, int rows_per_seq, const float* lse, const float* grad,
                              const z2z_listed_part& l, hipStream_t s);
int z2z_launch_listed(z2z_ctx* c, const int32_t* ids, long long rows, int per_row, const void* H, const void* W_base, const void* W_hyper,
                      const z2z_listed_part& part, hipStream_t s);
// Zeros in the listed columns of dZ, rows [r0, r0 + rows).
int z2z_launch_teacher_dz(z2z_ctx* c, const z2z_teacher& t, int r0, int rows, int rows_per_seq, void* base, size_t ld_base, void* hyper,
                          size_t ld_hyper, hipStream_t s);
int z2z_launch_extended_beam(z2z_ctx* c, const void* H, int32_t beams, const void* W_base, const void* W_hyper, const float* score,
                             int32_t picks, int32_t* parent, int32_t* code, float* picked, hipStream_t s);
// The pick from stored logits [B, V + cap] and the largest of each part of base_columns / hyper_columns columns (powers of two); the
// rows' log-sum-exps come from the parts' sums, or are given (part_s: nullptr).
int z2z_launch_beam_pick(z2z_ctx* c, const float* logits, const float* part_m, const float* part_s, int n_parts, int base_columns,
                         int hyper_columns, const float* row_lse, int beams, const float* score, int picks, int32_t* parent, int32_t* code, float* picked,
                         hipStream_t s);
int z2z_launch_part_max(z2z_ctx* c, const float* logits, float* part_m, int* n_parts, hipStream_t s);   // parts of 256 columns
int z2z_launch_codebook_reorder(z2z_ctx* c, int32_t beams, const int32_t* source, void* W_hyper, hipStream_t s);

// The layers' gated blocks where the encoder has them, else nullptr (an encoder with the flag is the first member of a z2z_gated_encoder).
inline const z2z_ffn* z2z_gated_layers(const z2z_encoder* enc) {
  return enc->attention_only == Z2Z_ENC_GATED ? reinterpret_cast<const z2z_gated_encoder*>(enc)->ffn : nullptr;
}
// The gated block's first product alone, and what its second is of: F [R, d_ff] and w [d, d_ff], bf16 or (group) in 4 bits.
struct z2z_ffn_out {
  void* F;
  const void *w, *scale;
  int group, d_ff;
  bool once, few, small;   // few, small: the second product runs on z2z_launch_few_linear, z2z_launch_small_linear
};
// What of a forward call on R rows is kept for its gradient (gated.h): nothing (all null), three matrices one behind the other in a buffer of 8 bytes an element
// of F, or (lo and f null) one of 4.
struct z2z_ffn_kept {
  uint16_t* f;
  uint32_t* hi;
  uint16_t* lo;
};
inline z2z_ffn_kept z2z_kept_in(void* p, size_t rows, int d_ff, int form = Z2Z_KEPT_32) {
  const size_t n = rows * d_ff;
  unsigned char* b = reinterpret_cast<unsigned char*>(p);
  if (!b) return z2z_ffn_kept{nullptr, nullptr, nullptr};
  if (form == Z2Z_KEPT_16) return z2z_ffn_kept{nullptr, reinterpret_cast<uint32_t*>(b), nullptr};
  return z2z_ffn_kept{reinterpret_cast<uint16_t*>(b), reinterpret_cast<uint32_t*>(b + 2 * n), reinterpret_cast<uint16_t*>(b + 6 * n)};
}
int z2z_launch_ffn_hidden(z2z_ctx* c, const void* X, const z2z_ffn* f, const z2z_ffn_kept& kept, int R, const int32_t* rows_dev, void* work, z2z_ffn_out* out,
                          hipStream_t s);
// The gated block on R rows (or the first *rows_dev of them), with work space of z2z_ffn_work bytes; stream_f32: residual and Y are fp32; kept: in the form that
// f->kept says, or nullptr.
size_t z2z_ffn_work(const z2z_ffn* f, int d, int rows);
int z2z_launch_ffn(z2z_ctx* c, const void* X, const z2z_ffn* f, const void* residual, void* Y, bool stream_f32, void* kept, int R, const int32_t* rows_dev,
                   void* work, hipStream_t s);
size_t z2z_ffn_backward_work(const z2z_ffn* f, int rows);
int z2z_launch_ffn_backward(z2z_ctx* c, const void* X, const z2z_ffn* f, const void* kept, const void* dY, void* dX, const z2z_ffn* grad, bool add, int R,
                            const int32_t* rows_dev, void* work, hipStream_t s);
int z2z_launch_fill_zero(void* p, size_t bytes, void* q, size_t bytes_q, hipStream_t s);   // multiples of 16
// 4-bit weights (q4.hip): from bf16, to bf16, and the product X w^T of few rows as fp32 parts [*ksplit][R][N], which the caller adds up before the next
// dense layer is launched
int z2z_launch_quantize_q4(const void* W, int rows, int cols, int group, void* q, void* scale, hipStream_t s);
int z2z_launch_expand_q4(const void* q, const void* scale, int rows, int cols, int group, void* W, hipStream_t s);
int z2z_launch_q4_parts(z2z_ctx* c, const void* X, const void* q, const void* scale, int group, int R, const int32_t* rows_dev, int N, int K,
                        const float** partial, int* ksplit, hipStream_t s);
int z2z_launch_clip_gradients(z2z_ctx* c, const z2z_gradient* g, int n, float max_norm, float* norm, hipStream_t s);

// At least `bytes` in the work buffer, every time a call is about to use it (Z2Z_ECAPTURE where it would have to grow under capture, Z2Z_ENOMEM where
// the device has no room: what was there is there still, or as much).  `at_least`: no less where it grows.
int z2z_work_reserve(z2z_ctx* c, z2z_work* w, size_t bytes, hipStream_t s, size_t at_least = 0);

// A work buffer that has to grow is freed and allocated again (hipFree / hipMalloc: the device synchronises that
// once).  A stream capture does not survive that, so under capture the call is refused instead, before anything
// is freed: the caller makes one eager call at the shape first.
inline int z2z_can_allocate(hipStream_t s) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &st) != hipSuccess) return Z2Z_EHIP;
  return st == hipStreamCaptureStatusNone ? Z2Z_OK : Z2Z_ECAPTURE;
}
#define Z2Z_TRY_GROW(s)                        \
  do {                                         \
    int _g = z2z_can_allocate(s);              \
    if (_g != Z2Z_OK) return _g;               \
  } while (0)

// A launch's threads are counted in 32 bits: beyond that the count wraps round, and fewer workgroups run, without an error.
constexpr long long kLaunchThreads = 0xFFFFFFFFLL;

// Device memory, or false.  A refusal is the call's to answer (another way, or Z2Z_ENOMEM): it does not stay behind as the runtime's last error,
// which the next launch, the program's too, would report as its own.
template <typename T>
inline bool z2z_device_malloc(T** p, size_t bytes) {
  if (hipMalloc(p, bytes) == hipSuccess) return true;
  *p = nullptr;
  (void)hipGetLastError();
  return false;
}

#define Z2Z_HIP_TRY(expr)                      \
  do {                                         \
    hipError_t _e = (expr);                    \
    if (_e != hipSuccess) return Z2Z_EHIP;     \
  } while (0)
