// C ABI of libz2z: argument checks, context life cycle, option and timing plumbing.
// Every entry point validates on the host, then hands over to a launcher; nothing here computes.
#include "z2z_internal.h"

#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "logits_common.h"
#include "logits_mid.h"

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Of n and m four-byte elements.
bool overlap(const void* p, long long n, const void* q, long long m) {
  const char *a = static_cast<const char*>(p), *b = static_cast<const char*>(q);
  return a && b && a < b + 4 * m && b < a + 4 * n;
}

// Of n and m bytes.
bool overlap_bytes(const void* p, size_t n, const void* q, size_t m) {
  const char *a = static_cast<const char*>(p), *b = static_cast<const char*>(q);
  return a && b && n && m && a < b + m && b < a + n;
}

void free_ctx(z2z_ctx* c) {
  if (!c) return;
  (void)hipFree(c->st.size);
  (void)hipFree(c->st.prev_code);
  (void)hipFree(c->st.prev_len);
  (void)hipFree(c->st.rounds);
  (void)hipFree(c->st.tail);
  (void)hipFree(c->st.ent_tokens);
  (void)hipFree(c->st.ent_len);
  (void)hipFree(c->st.slots);
  for (z2z_work* w : {&c->parts_ws, &c->draws_ws, &c->sample_ws, &c->enc_ws, &c->enc_bwd_ws, &c->bwd_ws, &c->partial_ws, &c->lookup_ws,
                      &c->ffn_ws, &c->clip_ws})
    (void)hipFree(w->p);
  (void)hipFree(c->coef_dev);
  (void)hipFree(c->prune_prefix);
  while (c->kept) {
    z2z_kept* k = c->kept;
    c->kept = k->next;
    (void)hipFree(k->p);
    delete k;
  }
  if (c->ev_created) {
    for (int i = 0; i < Z2Z_MAX_TIMED; ++i) {
      (void)hipEventDestroy(c->ev_start[i]);
      (void)hipEventDestroy(c->ev_stop[i]);
    }
  }
  delete c;
}

// (beyond this range the fp32 exponents of the softmax lose what they are to tell apart)
bool temperature_ok(float t) { return t >= 0.0625f && t <= 1024.0f; }

// At the start of every call that uses work buffers: whether it is captured into a graph (or may be: the runtime does not say).
void note_capture(z2z_ctx* c, hipStream_t s) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &st) == hipSuccess) {
    c->capturing = st != hipStreamCaptureStatusNone;
  } else {
    (void)hipGetLastError();
    c->capturing = true;
  }
}

// The same, on the context's device alone.
int enter(z2z_ctx* c, hipStream_t s) {
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess) return Z2Z_EHIP;
  if (device != c->device) return Z2Z_EINVAL;
  note_capture(c, s);
  return Z2Z_OK;
}

}  // namespace

int z2z_work_reserve(z2z_ctx* c, z2z_work* w, size_t bytes, hipStream_t s, size_t at_least) {
  if (bytes <= w->bytes) {
    w->named = w->named || c->capturing;
    return Z2Z_OK;
  }
  Z2Z_TRY_GROW(s);
  size_t want = std::max(bytes, at_least);
  if (w->named) {
    // What a graph names stays until z2z_destroy, the new memory is nobody's yet.  By half at least: with every length captured before the next one
    // asks for more, all that is kept is no more than twice the last buffer.
    want = std::max(want, w->bytes + w->bytes / 2);
    z2z_kept* k = new (std::nothrow) z2z_kept;
    void* p = nullptr;
    if (!k) return Z2Z_ENOMEM;
    if (!z2z_device_malloc(&p, want) && !z2z_device_malloc(&p, want = bytes)) {
      delete k;
      return Z2Z_ENOMEM;
    }
    k->p = w->p;
    k->next = c->kept;
    c->kept = k;
    w->p = p;
    w->bytes = want;
    w->named = c->capturing;
    return Z2Z_OK;
  }
  const size_t was = w->bytes;
  if (w->p) (void)hipFree(w->p);
  w->p = nullptr;
  w->bytes = 0;
  if (z2z_device_malloc(&w->p, want)) {
    w->bytes = want;
    w->named = c->capturing;
    return Z2Z_OK;
  }
  // (no room: smaller calls go on with what they had)
  if (was > 0 && z2z_device_malloc(&w->p, was)) w->bytes = was;
  return Z2Z_ENOMEM;
}

extern "C" {

Z2Z_API int z2z_create(z2z_ctx** out, const z2z_config* cfg) {
  if (!out || !cfg) return Z2Z_EINVAL;
  *out = nullptr;
  if (cfg->B < 1 || cfg->V < 1 || cfg->M < 1 || cfg->M > Z2Z_MAX_M) return Z2Z_EINVAL;
  if (cfg->cap < 0 || cfg->cap > Z2Z_MAX_CAP) return Z2Z_EINVAL;
  if ((long long)cfg->V + cfg->cap > (1LL << 24)) return Z2Z_EUNSUPPORTED;   // codes are packed in 24 bits
  if (cfg->dtype != Z2Z_F32 && cfg->dtype != Z2Z_BF16) return Z2Z_EUNSUPPORTED;
  if (cfg->pool != Z2Z_POOL_MEAN && cfg->pool != Z2Z_POOL_WEIGHTED) return Z2Z_EUNSUPPORTED;
  const int epc = cfg->dtype == Z2Z_BF16 ? 8 : 4;
  if (cfg->d < epc || cfg->d % epc != 0) return Z2Z_EINVAL;
  for (int j = 0; j < cfg->M; ++j)
    if (!isfinite(cfg->w[j])) return Z2Z_EINVAL;

  z2z_ctx* c = new (std::nothrow) z2z_ctx();
  if (!c) return Z2Z_ENOMEM;
  memset(c, 0, sizeof(*c));
  c->cfg = *cfg;
  if (hipGetDevice(&c->device) != hipSuccess) {
    delete c;
    return Z2Z_EHIP;
  }
  int lds = 0, cus = 0;
  if (hipDeviceGetAttribute(&lds, hipDeviceAttributeMaxSharedMemoryPerBlock, c->device) != hipSuccess) lds = 65536;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, c->device) != hipSuccess) cus = 256;
  c->lds_limit = lds > 160 * 1024 ? 160 * 1024 : lds;
  c->num_cu = cus;

  // pooling coefficients: coef[L][j] = 1/L or softmax(w[0..L))_j, computed in double
  for (int L = 1; L <= Z2Z_MAX_M; ++L) {
    double mx = -INFINITY, sum = 0.0;
    for (int j = 0; j < L; ++j) mx = cfg->w[j] > mx ? cfg->w[j] : mx;
    for (int j = 0; j < L; ++j) sum += exp((double)cfg->w[j] - mx);
    for (int j = 0; j < L; ++j)
      c->coef[L][j] = cfg->pool == Z2Z_POOL_MEAN ? (float)(1.0 / L) : (float)(exp((double)cfg->w[j] - mx) / sum);
  }

  LzwState& st = c->st;
  st.V = cfg->V;
  st.M = cfg->M;
  st.cap = cfg->cap;
  if (z2z_lzw_prepare(c) != Z2Z_OK) {   // sizes the hash table (st.nslots) for this device
    delete c;
    return Z2Z_EHIP;
  }
  const size_t B = (size_t)cfg->B;
  const size_t capn = cfg->cap > 0 ? (size_t)cfg->cap : 1;
  bool ok = true;
  ok = ok && z2z_device_malloc(&st.size, B * sizeof(int32_t));
  ok = ok && z2z_device_malloc(&st.prev_code, B * sizeof(int32_t));
  ok = ok && z2z_device_malloc(&st.prev_len, B * sizeof(int32_t));
  ok = ok && z2z_device_malloc(&st.rounds, B * sizeof(int32_t));
  ok = ok && z2z_device_malloc(&st.tail, 3 * B * sizeof(int32_t));
  ok = ok && hipMemset(st.rounds, 0, B * sizeof(int32_t)) == hipSuccess;
  ok = ok && z2z_device_malloc(&st.ent_tokens, B * capn * cfg->M * sizeof(int32_t));
  ok = ok && z2z_device_malloc(&st.ent_len, B * capn * sizeof(int32_t));
  ok = ok && z2z_device_malloc(&st.slots, B * (size_t)st.nslots * sizeof(unsigned long long));
  // fixed-size work buffers of calls that must not allocate on a stream: pruning's prefix map, and the pooling
  // coefficients on the device (the pooling's backward pass)
  ok = ok && z2z_device_malloc(&c->prune_prefix, B * capn * sizeof(int32_t));
  ok = ok && z2z_device_malloc(&c->coef_dev, sizeof(c->coef));
  ok = ok && hipMemcpy(c->coef_dev, c->coef, sizeof(c->coef), hipMemcpyHostToDevice) == hipSuccess;
  if (!ok) {
    free_ctx(c);
    return Z2Z_ENOMEM;
  }
  if (z2z_static_scratch_prepare(c) != Z2Z_OK) {   // the allocation-free entry point's array on this device
    free_ctx(c);
    return Z2Z_EHIP;
  }
  c->fast_ready = z2z_logits_fast_prepare(c) == Z2Z_OK;
  c->mid_ready = z2z_logits_mid_prepare(c) == Z2Z_OK;
  c->skinny_ready = z2z_logits_decode_prepare(c) == Z2Z_OK;      // the kernel itself; decode_ready: for this shape
  c->decode_ready = z2z_logits_decode_ok(c) && c->skinny_ready;
  c->trunc_ready = c->decode_ready && z2z_sample_truncated_prepare(c) == Z2Z_OK;
  if (z2z_launch_lzw_reset(c, nullptr) != Z2Z_OK ||
      hipStreamSynchronize(nullptr) != hipSuccess) {
    free_ctx(c);
    return Z2Z_EHIP;
  }
  *out = c;
  return Z2Z_OK;
}

Z2Z_API int z2z_destroy(z2z_ctx* ctx) {
  if (!ctx) return Z2Z_EINVAL;
  (void)hipDeviceSynchronize();
  free_ctx(ctx);
  return Z2Z_OK;
}

Z2Z_API int z2z_reset(z2z_ctx* ctx, void* stream) {
  if (!ctx) return Z2Z_EINVAL;
  return z2z_launch_lzw_reset(ctx, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_lzw_encode(z2z_ctx* ctx, const int32_t* d_tokens, const int32_t* d_lens, int32_t stride,
                           int32_t flags, int32_t* d_codes, int32_t* d_n_codes, int32_t out_stride,
                           int32_t* d_status, void* stream) {
  if (!ctx || !d_n_codes || !d_status) return Z2Z_EINVAL;
  if (stride < 0 || out_stride < 0) return Z2Z_EINVAL;
  if ((stride > 0 && !d_tokens) || (out_stride > 0 && !d_codes)) return Z2Z_EINVAL;
  if (flags != Z2Z_APPEND && flags != Z2Z_RESET) return Z2Z_EINVAL;
  return z2z_launch_lzw_encode(ctx, d_tokens, d_lens, stride, flags, d_codes, d_n_codes, out_stride, d_status,
                               static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_lzw_decode(z2z_ctx* ctx, const int32_t* d_codes, const int32_t* d_n_codes, int32_t stride,
                           int32_t flags, int32_t* d_tokens, int32_t* d_n_tokens, int32_t out_stride,
                           int32_t* d_status, void* stream) {
  if (!ctx || !d_n_tokens || !d_status) return Z2Z_EINVAL;
  if (stride < 0 || out_stride < 0) return Z2Z_EINVAL;
  if (stride > 0 && !d_codes) return Z2Z_EINVAL;
  if (out_stride > 0 && !d_tokens) return Z2Z_EINVAL;
  if (out_stride == 0 && d_tokens) return Z2Z_EINVAL;
  if (flags != Z2Z_APPEND && flags != Z2Z_RESET) return Z2Z_EINVAL;
  return z2z_launch_lzw_decode(ctx, d_codes, d_n_codes, stride, flags, d_tokens, d_n_tokens, out_stride, d_status,
                               static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_codebook(z2z_ctx* ctx, const int32_t** d_entries, const int32_t** d_entry_len,
                         const int32_t** d_size) {
  if (!ctx) return Z2Z_EINVAL;
  if (d_entries) *d_entries = ctx->st.ent_tokens;
  if (d_entry_len) *d_entry_len = ctx->st.ent_len;
  if (d_size) *d_size = ctx->st.size;
  return Z2Z_OK;
}

Z2Z_API int z2z_step_update(z2z_ctx* ctx, const int32_t* d_codes, int32_t stride, const void* d_E, void* d_W_hyper,
                            int32_t* d_n_tokens, int32_t* d_status, void* stream) {
  if (!ctx || !d_codes || !d_n_tokens || !d_status || stride < 1) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && (!d_E || !d_W_hyper)) return Z2Z_EINVAL;
  if (!aligned16(d_E) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  return z2z_launch_step_update(ctx, d_codes, stride, d_E, d_W_hyper, d_n_tokens, d_status,
                                static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_lzw_rounds(z2z_ctx* ctx, const int32_t** d_rounds) {
  if (!ctx || !d_rounds) return Z2Z_EINVAL;
  *d_rounds = ctx->st.rounds;
  return Z2Z_OK;
}

Z2Z_API int z2z_codebook_usage(z2z_ctx* ctx, const int32_t* d_codes, const int32_t* d_n_codes, int32_t stride,
                               int32_t* d_usage, void* stream) {
  if (!ctx || stride < 0 || (stride > 0 && !d_codes)) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_usage) return Z2Z_EINVAL;
  if (ctx->cfg.cap == 0 || stride == 0) return Z2Z_OK;
  return z2z_launch_codebook_usage(ctx, d_codes, d_n_codes, stride, d_usage, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_codebook_prune(z2z_ctx* ctx, const int32_t* d_keep, int32_t* d_new_id, int32_t* d_n_kept,
                               void* stream) {
  if (!ctx || !d_n_kept) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && (!d_keep || !d_new_id)) return Z2Z_EINVAL;
  return z2z_launch_codebook_prune(ctx, d_keep, d_new_id, d_n_kept, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_codebook_prefill(z2z_ctx* ctx, const int32_t* d_phrases, const int32_t* d_phrase_len,
                                 const int32_t* d_counts, int32_t n_max, int32_t flags, int32_t* d_n_added,
                                 int32_t* d_status, void* stream) {
  if (!ctx || !d_n_added || !d_status || n_max < 0) return Z2Z_EINVAL;
  if (n_max > 0 && (!d_phrases || !d_phrase_len)) return Z2Z_EINVAL;
  if (flags != Z2Z_RESET && flags != Z2Z_APPEND) return Z2Z_EINVAL;
  return z2z_launch_codebook_prefill(ctx, d_phrases, d_phrase_len, d_counts, n_max, flags, d_n_added, d_status,
                                     static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_hyper_embed(z2z_ctx* ctx, const void* d_E, void* d_W_hyper, const int32_t* d_first,
                            int32_t max_new, void* stream) {
  if (!ctx || !d_E) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (!aligned16(d_E) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  return z2z_launch_hyper_embed(ctx, d_E, d_W_hyper, d_first, max_new, static_cast<hipStream_t>(stream));
}

namespace {

// of a gated block on a context of width d: its description's numbers, and its pointers
int ffn_ok(const z2z_ctx* c, const z2z_ffn* f, bool bf16_only) {
  if (!f || f->d_ff < 1 || (f->kept != Z2Z_KEPT_32 && f->kept != Z2Z_KEPT_16) || (f->act != Z2Z_ACT_SILU && f->act != Z2Z_ACT_GELU)) return Z2Z_EINVAL;
  if (!f->w_1 || !f->w_2 || !aligned16(f->w_1) || !aligned16(f->w_2)) return Z2Z_EINVAL;
  if (f->group != 0 && f->group != 32 && f->group != 64 && f->group != 128) return Z2Z_EINVAL;
  if (f->group != 0 && (!f->scale_1 || !f->scale_2 || !aligned16(f->scale_1) || !aligned16(f->scale_2))) return Z2Z_EINVAL;
  const int d = c->cfg.d;
  if (c->cfg.dtype != Z2Z_BF16 || !c->fast_ready || d % 64 != 0 || f->d_ff % 64 != 0) return Z2Z_EUNSUPPORTED;
  // (offsets of 32 bits: in a projection, and in 256 rows of dG | dU, whose products read them from the first of these on; no launch has 2^32 threads then)
  if (((long long)f->d_ff + 128) * d * 2 >= (1LL << 31) || 256LL * 4 * f->d_ff >= (1LL << 32)) return Z2Z_EUNSUPPORTED;
  if (f->group != 0 && (bf16_only || d % f->group != 0 || f->d_ff % f->group != 0)) return Z2Z_EUNSUPPORTED;
  return Z2Z_OK;
}

// every pointer a layer of the description must carry, present and 16-byte aligned; kind: attention_only of the encoder, or of the one whose gradients it names
bool encoder_pointers_ok(const z2z_encoder* enc, int32_t kind) {
  if (!enc || !enc->layers) return false;
  if (enc->n_layers < 1 || enc->n_layers > Z2Z_MAX_ENCODER_LAYERS) return false;
  if (!aligned16(enc->pos)) return false;
  for (int l = 0; l < enc->n_layers; ++l) {
    const z2z_encoder_layer& y = enc->layers[l];
    const void* always[] = {y.ln1_g, y.ln1_b, y.w_qkv, y.b_qkv, y.w_o, y.b_o};
    for (const void* p : always)
      if (!p || !aligned16(p)) return false;
    if (kind == Z2Z_ENC_GATED) {
      const z2z_ffn* f = z2z_gated_layers(enc);
      const void* ffn[] = {y.ln2_g, y.ln2_b, f ? f[l].w_1 : nullptr, f ? f[l].w_2 : nullptr};
      for (const void* p : ffn)
        if (!p || !aligned16(p)) return false;
    } else if (!kind) {
      const void* ffn[] = {y.ln2_g, y.ln2_b, y.w_1, y.b_1, y.w_2, y.b_2};
      for (const void* p : ffn)
        if (!p || !aligned16(p)) return false;
    }
  }
  return true;
}

bool encoder_ok(const z2z_encoder* enc) { return enc && encoder_pointers_ok(enc, enc->attention_only); }

// the rest of a description with gated blocks; training: over bf16 weights
int gated_layers_ok(const z2z_ctx* c, const z2z_encoder* enc, bool training) {
  const z2z_ffn* f = z2z_gated_layers(enc);
  for (int l = 0; f && l < enc->n_layers; ++l) {
    const int rc = ffn_ok(c, f + l, training);
    if (rc != Z2Z_OK) return rc;
    if (f[l].d_ff != f[0].d_ff || f[l].kept != Z2Z_KEPT_32) return Z2Z_EINVAL;
  }
  return Z2Z_OK;
}

}  // namespace

Z2Z_API int z2z_hyper_encode(z2z_ctx* ctx, const void* d_E, const z2z_encoder* enc, void* d_W_hyper,
                             const int32_t* d_first, int32_t max_new, void* stream) {
  if (!ctx || !d_E || !encoder_ok(enc)) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (!aligned16(d_E) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  if (!z2z_hyper_encode_ok(ctx, enc)) return Z2Z_EUNSUPPORTED;
  const int ok = gated_layers_ok(ctx, enc, false);
  if (ok != Z2Z_OK) return ok;
  note_capture(ctx, static_cast<hipStream_t>(stream));
  return z2z_launch_hyper_encode(ctx, d_E, enc, d_W_hyper, d_first, max_new, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_hyper_encode_keep(z2z_ctx* ctx, const void* d_E, const z2z_encoder* enc, void* d_W_hyper, void* stream) {
  if (!ctx || !d_E || !encoder_ok(enc)) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (!aligned16(d_E) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  if (!z2z_hyper_encode_ok(ctx, enc)) return Z2Z_EUNSUPPORTED;
  const int ok = gated_layers_ok(ctx, enc, true);
  if (ok != Z2Z_OK) return ok;
  note_capture(ctx, static_cast<hipStream_t>(stream));
  return z2z_launch_hyper_encode_train(ctx, 1, d_E, enc, d_W_hyper, nullptr, nullptr, nullptr,
                                       static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_hyper_encode_backward(z2z_ctx* ctx, const void* d_E, const z2z_encoder* enc, const void* d_dW_hyper,
                                      const z2z_encoder* grad, float* d_dE, int32_t flags, void* stream) {
  if (!ctx || !d_E || !d_dE || !encoder_ok(enc) || !grad) return Z2Z_EINVAL;
  if (enc->attention_only == Z2Z_ENC_GATED && grad->attention_only != Z2Z_ENC_GATED) return Z2Z_EINVAL;
  if (!encoder_pointers_ok(grad, enc->attention_only)) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_dW_hyper) return Z2Z_EINVAL;
  if (grad->n_layers != enc->n_layers || (enc->pos && !grad->pos)) return Z2Z_EINVAL;
  if (flags & ~Z2Z_ENC_KEPT) return Z2Z_EINVAL;
  if (!aligned16(d_E) || !aligned16(d_dW_hyper) || !aligned16(d_dE)) return Z2Z_EINVAL;
  if (!z2z_hyper_encode_ok(ctx, enc)) return Z2Z_EUNSUPPORTED;
  const int ok = gated_layers_ok(ctx, enc, true);
  if (ok != Z2Z_OK) return ok;
  note_capture(ctx, static_cast<hipStream_t>(stream));
  return z2z_launch_hyper_encode_train(ctx, (flags & Z2Z_ENC_KEPT) ? 2 : 0, d_E, enc, nullptr, d_dW_hyper, grad, d_dE,
                                       static_cast<hipStream_t>(stream));
}

namespace {

constexpr int32_t kFfnRows = 1 << 22;

struct Bytes {
  const void* p;
  size_t n;
};
// Whether anything that is written overlaps anything that is read, or the rest of what is written.
bool clashes(const Bytes* in, int n_in, const Bytes* out, int n_out) {
  for (int i = 0; i < n_out; ++i) {
    for (int k = 0; k < n_in; ++k)
      if (overlap_bytes(out[i].p, out[i].n, in[k].p, in[k].n)) return true;
    for (int k = 0; k < i; ++k)
      if (overlap_bytes(out[i].p, out[i].n, out[k].p, out[k].n)) return true;
  }
  return false;
}

// Bytes of a matrix of 4-bit weights as quantize_q4 writes them.
size_t q4_bytes(size_t rows, size_t cols) { return rows * ((cols + 127) / 128) * 64; }

struct FfnBytes {
  size_t w_1, w_2, scale_1, scale_2;
};
// ... of what is kept of a call
size_t kept_bytes(const z2z_ffn* f, int32_t rows) { return (size_t)rows * f->d_ff * (f->kept == Z2Z_KEPT_16 ? 4 : 8); }
FfnBytes ffn_bytes(const z2z_ctx* c, const z2z_ffn* f) {
  const size_t d = c->cfg.d, n = f->d_ff;
  if (!f->group) return FfnBytes{4 * n * d, 2 * n * d, 0, 0};
  return FfnBytes{q4_bytes(2 * n, d), q4_bytes(d, n), 4 * n * d / f->group, 2 * n * d / f->group};
}

}  // namespace

Z2Z_API int z2z_gated_ffn(z2z_ctx* ctx, const void* d_X, int32_t rows, const z2z_ffn* ffn, const void* d_residual, void* d_Y, void* d_kept,
                          void* stream) {
  if (!ctx || rows < 0 || (rows > 0 && (!d_X || !d_Y))) return Z2Z_EINVAL;
  if (!aligned16(d_X) || !aligned16(d_residual) || !aligned16(d_Y) || !aligned16(d_kept)) return Z2Z_EINVAL;
  int rc = ffn_ok(ctx, ffn, d_kept != nullptr);
  if (rc != Z2Z_OK) return rc;
  if (rows > kFfnRows) return Z2Z_EUNSUPPORTED;
  const size_t row = (size_t)rows * ctx->cfg.d * 2, kept = kept_bytes(ffn, rows);
  const FfnBytes w = ffn_bytes(ctx, ffn);
  const Bytes in[] = {{d_X, row}, {d_residual == d_Y ? nullptr : d_residual, row}, {ffn->w_1, w.w_1}, {ffn->w_2, w.w_2}, {ffn->scale_1, w.scale_1}, {ffn->scale_2, w.scale_2}};
  const Bytes out[] = {{d_Y, row}, {d_kept, kept}};
  if (clashes(in, 6, out, 2) || overlap_bytes(d_kept, kept, d_residual, row)) return Z2Z_EINVAL;
  rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK || rows == 0) return rc;
  if (!d_kept || ffn->kept != Z2Z_KEPT_32) {       // (else F is a part of what is kept, and weights that would be expanded keep nothing)
    rc = z2z_work_reserve(ctx, &ctx->ffn_ws, z2z_ffn_work(ffn, ctx->cfg.d, rows), static_cast<hipStream_t>(stream));
    if (rc != Z2Z_OK) return rc;
  }
  return z2z_launch_ffn(ctx, d_X, ffn, d_residual, d_Y, false, d_kept, rows, nullptr, ctx->ffn_ws.p, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_gated_ffn_backward(z2z_ctx* ctx, const void* d_X, int32_t rows, const z2z_ffn* ffn, const void* d_kept, const void* d_dY, void* d_dX,
                                   const z2z_ffn* grad, int32_t flags, void* stream) {
  if (!ctx || rows < 0 || (rows > 0 && (!d_X || !d_kept || !d_dY || !d_dX))) return Z2Z_EINVAL;
  if (flags != 0 && flags != Z2Z_GRAD_ADD) return Z2Z_EINVAL;
  if (!aligned16(d_X) || !aligned16(d_kept) || !aligned16(d_dY) || !aligned16(d_dX)) return Z2Z_EINVAL;
  if (!grad || !grad->w_1 || !grad->w_2 || !aligned16(grad->w_1) || !aligned16(grad->w_2)) return Z2Z_EINVAL;
  int rc = ffn_ok(ctx, ffn, true);
  if (rc != Z2Z_OK) return rc;
  if (rows > kFfnRows) return Z2Z_EUNSUPPORTED;
  const size_t row = (size_t)rows * ctx->cfg.d * 2, kept = kept_bytes(ffn, rows);
  const FfnBytes w = ffn_bytes(ctx, ffn);
  const size_t w1 = w.w_1, w2 = w.w_2;
  const Bytes in[] = {{d_X, row}, {d_kept, kept}, {d_dY, row}, {ffn->w_1, w1}, {ffn->w_2, w2}}, out[] = {{d_dX, row}, {grad->w_1, w1}, {grad->w_2, w2}};
  if (clashes(in, 5, out, 3)) return Z2Z_EINVAL;
  rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (rows == 0) return flags == Z2Z_GRAD_ADD ? Z2Z_OK : z2z_launch_fill_zero(const_cast<void*>(grad->w_1), w1, const_cast<void*>(grad->w_2), w2, s);
  rc = z2z_work_reserve(ctx, &ctx->ffn_ws, z2z_ffn_backward_work(ffn, rows), s);
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_ffn_backward(ctx, d_X, ffn, d_kept, d_dY, d_dX, grad, flags == Z2Z_GRAD_ADD, rows, nullptr, ctx->ffn_ws.p, s);
}

Z2Z_API int z2z_quantize_q4(z2z_ctx* ctx, const void* d_W, int32_t rows, int32_t cols, int32_t group, void* d_q, void* d_scale, void* stream) {
  if (!ctx || rows < 1 || cols < 1 || !d_W || !d_q || !d_scale) return Z2Z_EINVAL;
  if (!aligned16(d_W) || !aligned16(d_q) || !aligned16(d_scale)) return Z2Z_EINVAL;
  if (group != 32 && group != 64 && group != 128) return Z2Z_EINVAL;
  if (ctx->cfg.dtype != Z2Z_BF16 || rows % 16 != 0 || cols % 64 != 0 || cols % group != 0) return Z2Z_EUNSUPPORTED;
  const size_t n = (size_t)rows * cols, q = q4_bytes(rows, cols), sc = n / group * 2;
  if (overlap_bytes(d_q, q, d_W, 2 * n) || overlap_bytes(d_scale, sc, d_W, 2 * n) || overlap_bytes(d_q, q, d_scale, sc)) return Z2Z_EINVAL;
  const int rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_quantize_q4(d_W, rows, cols, group, d_q, d_scale, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_clip_gradients(z2z_ctx* ctx, const z2z_gradient* gradients, int32_t n, float max_norm, float* d_norm, void* stream) {
  if (!ctx || n < 0 || (n > 0 && !gradients) || !d_norm || !(max_norm >= 0.f)) return Z2Z_EINVAL;      // (a NaN, too)
  if (reinterpret_cast<uintptr_t>(d_norm) & 3u) return Z2Z_EINVAL;
  for (int32_t i = 0; i < n; ++i) {
    const z2z_gradient& g = gradients[i];
    if (g.n < 0 || (g.n > 0 && !g.data) || (g.dtype != Z2Z_F32 && g.dtype != Z2Z_BF16) || g.reserved != 0) return Z2Z_EINVAL;
    const uintptr_t size = g.dtype == Z2Z_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(g.data) % size != 0 || reinterpret_cast<uintptr_t>(g.out) % size != 0) return Z2Z_EINVAL;
  }
  if (n > Z2Z_MAX_GRADIENTS) return Z2Z_EUNSUPPORTED;
  const int rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_clip_gradients(ctx, gradients, n, max_norm, d_norm, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_extended_logits(z2z_ctx* ctx, const void* d_H, int32_t rows, int32_t rows_per_seq,
                                const void* d_W_base, const void* d_W_hyper, int32_t* d_argmax, float* d_max,
                                float* d_lse, float* d_logits, void* stream) {
  if (!ctx || !d_H || !d_W_base) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (rows_per_seq < 1 || rows < 1) return Z2Z_EINVAL;
  if ((long long)rows_per_seq * ctx->cfg.B != (long long)rows) return Z2Z_EINVAL;
  if (!aligned16(d_H) || !aligned16(d_W_base) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  note_capture(ctx, static_cast<hipStream_t>(stream));
  return z2z_launch_extended_logits(ctx, d_H, rows, rows_per_seq, d_W_base, d_W_hyper, d_argmax, d_max, d_lse,
                                    d_logits, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_extended_logits_static(z2z_ctx* ctx, const void* d_H, int32_t rows, int32_t rows_per_seq,
                                       const void* d_W_base, const void* d_W_hyper, int32_t* d_argmax,
                                       float* d_max, float* d_lse, float* d_logits, void* stream) {
  if (!ctx || !d_H || !d_W_base) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (rows_per_seq < 1 || rows < 1) return Z2Z_EINVAL;
  if ((long long)rows_per_seq * ctx->cfg.B != (long long)rows) return Z2Z_EINVAL;
  if (!aligned16(d_H) || !aligned16(d_W_base) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  return z2z_launch_extended_logits(ctx, d_H, rows, rows_per_seq, d_W_base, d_W_hyper, d_argmax, d_max, d_lse,
                                    d_logits, static_cast<hipStream_t>(stream), true);
}

Z2Z_API int z2z_extended_sample(z2z_ctx* ctx, const void* d_H, int32_t rows, int32_t rows_per_seq,
                                const void* d_W_base, const void* d_W_hyper, float temperature, int32_t top_k,
                                float top_p, uint64_t seed, uint64_t step, int32_t* d_token, float* d_logprob,
                                void* stream) {
  if (!ctx || !d_H || !d_W_base || !d_token) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (rows_per_seq < 1 || rows < 1) return Z2Z_EINVAL;
  if ((long long)rows_per_seq * ctx->cfg.B != (long long)rows) return Z2Z_EINVAL;
  if (!(temperature > 0.f) || !(temperature < 3.0e38f)) return Z2Z_EINVAL;
  if (!(top_p > 0.f)) return Z2Z_EINVAL;          // also rejects NaN; >= 1 switches the filter off
  if (!aligned16(d_H) || !aligned16(d_W_base) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  note_capture(ctx, static_cast<hipStream_t>(stream));
  return z2z_launch_extended_sample(ctx, d_H, rows, rows_per_seq, d_W_base, d_W_hyper, temperature, top_k, top_p,
                                    seed, step, d_token, d_logprob, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_embed_codes(z2z_ctx* ctx, const int32_t* d_codes, const int32_t* d_n_codes, int32_t stride, const void* d_E,
                            const void* d_W_hyper, float scale, void* d_X, int32_t* d_status, void* stream) {
  if (!ctx || !d_E || !d_status || stride < 0) return Z2Z_EINVAL;
  if (stride > 0 && (!d_codes || !d_X)) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (overlap(d_status, ctx->cfg.B, d_n_codes, ctx->cfg.B)) return Z2Z_EINVAL;   // (other workgroups read the lengths while the statuses are written)
  if (!isfinite(scale)) return Z2Z_EINVAL;
  if (!aligned16(d_E) || !aligned16(d_W_hyper) || !aligned16(d_X)) return Z2Z_EINVAL;
  const int rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_embed_codes(ctx, d_codes, d_n_codes, stride, d_E, d_W_hyper, scale, d_X, d_status,
                                static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_embed_codes_backward(z2z_ctx* ctx, const int32_t* d_codes, const int32_t* d_n_codes, int32_t stride, float scale,
                                     const void* d_dX, int32_t flags, float* d_dE, void* d_dW_hyper, void* stream) {
  if (!ctx || !d_dE || stride < 0) return Z2Z_EINVAL;
  if (stride > 0 && (!d_codes || !d_dX)) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_dW_hyper) return Z2Z_EINVAL;
  if (flags != 0 && flags != Z2Z_GRAD_ADD) return Z2Z_EINVAL;
  if (!isfinite(scale)) return Z2Z_EINVAL;
  if (!aligned16(d_dX) || !aligned16(d_dE) || !aligned16(d_dW_hyper)) return Z2Z_EINVAL;
  const int rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_embed_codes_backward(ctx, d_codes, d_n_codes, stride, scale, d_dX, flags, d_dE, d_dW_hyper,
                                         static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_extended_beam(z2z_ctx* ctx, const void* d_H, int32_t rows, int32_t beams, const void* d_W_base, const void* d_W_hyper,
                              const float* d_score, int32_t n_pick, int32_t* d_parent, int32_t* d_code, float* d_picked, void* stream) {
  if (!ctx || !d_H || !d_W_base || !d_score || !d_parent || !d_code || !d_picked) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (rows != ctx->cfg.B || beams < 1 || rows % beams != 0 || n_pick < 1) return Z2Z_EINVAL;
  if (beams > Z2Z_MAX_BEAMS || n_pick > Z2Z_MAX_PICK) return Z2Z_EUNSUPPORTED;
  if (overlap(d_score, rows, d_picked, (long long)(rows / beams) * n_pick) && (d_picked != d_score || n_pick != beams))
    return Z2Z_EINVAL;                               // (other prompts' scores would be written over)
  if (!aligned16(d_H) || !aligned16(d_W_base) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  const int rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_extended_beam(ctx, d_H, beams, d_W_base, d_W_hyper, d_score, n_pick, d_parent, d_code, d_picked,
                                  static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_codebook_reorder(z2z_ctx* ctx, int32_t beams, const int32_t* d_source, void* d_W_hyper, void* stream) {
  if (!ctx || !d_source || beams < 1 || ctx->cfg.B % beams != 0) return Z2Z_EINVAL;
  if (beams > Z2Z_MAX_BEAMS) return Z2Z_EUNSUPPORTED;
  if (!aligned16(d_W_hyper)) return Z2Z_EINVAL;
  const int rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK) return rc;
  return z2z_launch_codebook_reorder(ctx, beams, d_source, d_W_hyper, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_extended_nll(z2z_ctx* ctx, const void* d_H, int32_t rows, int32_t rows_per_seq, const void* d_W_base,
                             const void* d_W_hyper, const int32_t* d_targets, float* d_nll, float* d_lse,
                             void* stream) {
  if (!ctx || !d_H || !d_W_base || !d_targets || !d_nll || !d_lse) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (rows_per_seq < 1 || rows < 1) return Z2Z_EINVAL;
  if ((long long)rows_per_seq * ctx->cfg.B != (long long)rows) return Z2Z_EINVAL;
  if (!aligned16(d_H) || !aligned16(d_W_base) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  note_capture(ctx, static_cast<hipStream_t>(stream));
  return z2z_launch_extended_nll(ctx, d_H, rows, rows_per_seq, d_W_base, d_W_hyper, d_targets, d_nll, d_lse,
                                 static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_extended_nll_backward(z2z_ctx* ctx, const void* d_H, int32_t rows, int32_t rows_per_seq,
                                      const void* d_W_base, const void* d_W_hyper, const int32_t* d_targets,
                                      const float* d_lse, const float* d_grad_nll, void* d_dH, void* d_dW_base,
                                      void* d_dW_hyper, void* stream) {
  if (!ctx || !d_H || !d_W_base || !d_targets || !d_lse || !d_dH || !d_dW_base) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && (!d_W_hyper || !d_dW_hyper)) return Z2Z_EINVAL;
  if (rows_per_seq < 1 || rows < 1) return Z2Z_EINVAL;
  if ((long long)rows_per_seq * ctx->cfg.B != (long long)rows) return Z2Z_EINVAL;
  if (!aligned16(d_H) || !aligned16(d_W_base) || !aligned16(d_W_hyper) || !aligned16(d_dH) || !aligned16(d_dW_base) ||
      !aligned16(d_dW_hyper))
    return Z2Z_EINVAL;
  note_capture(ctx, static_cast<hipStream_t>(stream));
  return z2z_launch_extended_nll_backward(ctx, d_H, rows, rows_per_seq, d_W_base, d_W_hyper, d_targets, d_lse,
                                          d_grad_nll, d_dH, d_dW_base, d_dW_hyper, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_extended_distill(z2z_ctx* ctx, const void* d_H, int32_t rows, int32_t rows_per_seq, const void* d_W_base,
                                 const void* d_W_hyper, int32_t n_teacher, const int32_t* d_ids, const float* d_teacher,
                                 float temperature, float* d_kl, float* d_lse, float* d_student, void* stream) {
  if (!ctx || !d_H || !d_W_base || !d_ids || !d_teacher || !d_kl || !d_lse || !d_student) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_W_hyper) return Z2Z_EINVAL;
  if (rows_per_seq < 1 || rows < 1 || n_teacher < 1) return Z2Z_EINVAL;
  if ((long long)rows_per_seq * ctx->cfg.B != (long long)rows) return Z2Z_EINVAL;
  if (d_student == d_teacher || (const void*)d_student == d_ids) return Z2Z_EINVAL;      // (written before the teacher is read)
  if (!temperature_ok(temperature)) return Z2Z_EINVAL;
  if (!aligned16(d_H) || !aligned16(d_W_base) || !aligned16(d_W_hyper)) return Z2Z_EINVAL;
  if (n_teacher > Z2Z_MAX_TEACHER) return Z2Z_EUNSUPPORTED;
  const int rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK) return rc;
  const z2z_teacher t = {n_teacher, d_ids, d_teacher, temperature, nullptr};
  return z2z_launch_extended_distill(ctx, d_H, rows, rows_per_seq, d_W_base, d_W_hyper, t, d_kl, d_lse, d_student,
                                     static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_extended_distill_backward(z2z_ctx* ctx, const void* d_H, int32_t rows, int32_t rows_per_seq, const void* d_W_base,
                                          const void* d_W_hyper, int32_t n_teacher, const int32_t* d_ids, const float* d_teacher,
                                          float temperature, const float* d_lse, const float* d_student, const float* d_grad_kl,
                                          void* d_dH, void* d_dW_base, void* d_dW_hyper, void* stream) {
  if (!ctx || !d_H || !d_W_base || !d_ids || !d_teacher || !d_lse || !d_student || !d_dH || !d_dW_base) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && (!d_W_hyper || !d_dW_hyper)) return Z2Z_EINVAL;
  if (rows_per_seq < 1 || rows < 1 || n_teacher < 1) return Z2Z_EINVAL;
  if ((long long)rows_per_seq * ctx->cfg.B != (long long)rows) return Z2Z_EINVAL;
  if (!temperature_ok(temperature)) return Z2Z_EINVAL;
  if (!aligned16(d_H) || !aligned16(d_W_base) || !aligned16(d_W_hyper) || !aligned16(d_dH) || !aligned16(d_dW_base) ||
      !aligned16(d_dW_hyper))
    return Z2Z_EINVAL;
  if (n_teacher > Z2Z_MAX_TEACHER) return Z2Z_EUNSUPPORTED;
  const int rc = enter(ctx, static_cast<hipStream_t>(stream));
  if (rc != Z2Z_OK) return rc;
  const z2z_teacher t = {n_teacher, d_ids, d_teacher, temperature, d_student};
  return z2z_launch_extended_nll_backward(ctx, d_H, rows, rows_per_seq, d_W_base, d_W_hyper, nullptr, d_lse, d_grad_kl, d_dH, d_dW_base,
                                          d_dW_hyper, static_cast<hipStream_t>(stream), &t);
}

Z2Z_API int z2z_hyper_embed_backward(z2z_ctx* ctx, const void* d_dW_hyper, float* d_dE, void* stream) {
  if (!ctx || !d_dE) return Z2Z_EINVAL;
  if (ctx->cfg.cap > 0 && !d_dW_hyper) return Z2Z_EINVAL;
  if (ctx->cfg.dtype != Z2Z_BF16) return Z2Z_EUNSUPPORTED;
  return z2z_launch_hyper_embed_backward(ctx, d_dW_hyper, d_dE, static_cast<hipStream_t>(stream));
}

Z2Z_API int z2z_set_option(z2z_ctx* ctx, int32_t key, int32_t value) {
  if (!ctx) return Z2Z_EINVAL;
  switch (key) {
    case Z2Z_OPT_LOGITS_KERNEL: ctx->opt_logits_kernel = value; return Z2Z_OK;
    case Z2Z_OPT_LOGITS_STRIP:
      if (value < 0) return Z2Z_EINVAL;
      ctx->opt_logits_strip = value;
      return Z2Z_OK;
    case Z2Z_OPT_LZW_KERNEL: ctx->opt_lzw_kernel = value; return Z2Z_OK;
    case Z2Z_OPT_DECODE_KERNEL: ctx->opt_decode_kernel = value; return Z2Z_OK;
    case Z2Z_OPT_SAMPLE_KERNEL: ctx->opt_sample_kernel = value; return Z2Z_OK;
    case Z2Z_OPT_BACKWARD_CHUNK:
      if (value < 0) return Z2Z_EINVAL;
      ctx->opt_backward_chunk = value;
      return Z2Z_OK;
    case Z2Z_OPT_LOGITS_MAP:
      if (value != 0 && ((value & 0xFF) < 1 || ((value >> 8) & 0xFF) < 1 || ((value >> 16) & 0xFF) < 1 ||
                         ((value >> 24) & 0xFF) < 1 || ((value >> 16) & 0xFF) * ((value >> 24) & 0xFF) != 8))
        return Z2Z_EINVAL;
      ctx->opt_logits_map = value;
      return Z2Z_OK;
    case Z2Z_OPT_TIMING:
      if (value && !ctx->ev_created) {
        for (int i = 0; i < Z2Z_MAX_TIMED; ++i) {
          if (hipEventCreate(&ctx->ev_start[i]) != hipSuccess || hipEventCreate(&ctx->ev_stop[i]) != hipSuccess)
            return Z2Z_EHIP;
        }
        ctx->ev_created = 1;
      }
      ctx->opt_timing = value ? 1 : 0;
      return Z2Z_OK;
    default: return Z2Z_EINVAL;
  }
}

Z2Z_API int z2z_read_timing(z2z_ctx* ctx, float* total_ms, int32_t* launches) {
  if (!ctx || !total_ms || !launches) return Z2Z_EINVAL;
  float sum = 0.f;
  for (int i = 0; i < ctx->n_timed; ++i) {
    if (hipEventSynchronize(ctx->ev_stop[i]) != hipSuccess) return Z2Z_EHIP;
    float ms = 0.f;
    if (hipEventElapsedTime(&ms, ctx->ev_start[i], ctx->ev_stop[i]) != hipSuccess) return Z2Z_EHIP;
    sum += ms;
  }
  *total_ms = sum;
  *launches = ctx->n_timed;
  ctx->n_timed = 0;
  return Z2Z_OK;
}

Z2Z_API int z2z_read_launches(const z2z_ctx* ctx, int64_t* counts) {
  if (!ctx || !counts) return Z2Z_EINVAL;
  for (int i = 0; i < Z2Z_N_KERNEL_FAMILIES; ++i) counts[i] = ctx->n_launch[i];
  return Z2Z_OK;
}

Z2Z_API const char* z2z_strerror(int code) {
  switch (code) {
    case Z2Z_OK: return "ok";
    case Z2Z_EINVAL: return "invalid argument";
    case Z2Z_ENOMEM: return "out of device or host memory";
    case Z2Z_EHIP: return "HIP runtime error";
    case Z2Z_EUNSUPPORTED: return "unsupported dtype or pooling kind";
    case Z2Z_ELIMIT: return "beyond the fixed scratch size of the allocation-free entry point";
    case Z2Z_ECAPTURE: return "a work buffer would have to grow while the stream is being captured";
    default: return "unknown error";
  }
}

}  // extern "C"
