// Beam search over the extended vocabulary (gfx950): the pick over a prompt's beams and all their columns, and the move of
// the beams' codebooks that follows it.
//
// Section 2.3 of the zip2zip paper, step 9, picks from the joint distribution over base tokens and hypertokens; here the pick
// is that of a beam search: of all continuations (beam r, column v) of a prompt the n_pick best by
//   score[r] + logit[r, v] - lse[r],
// equal ones by lower beam, then lower column.  A beam's codebook belongs to its history ("Consistent Vocabulary Updates"), so a
// beam that goes on from another one takes over its codebook and cache rows.
#include "logits_common.h"

#include <string.h>

#include <algorithm>

namespace {

using namespace z2z_logits;

// ---- the pick -----------------------------------------------------------------------------------------------------------------
struct PickArgs {
  const float* logits;      // [rows, ld]
  const float* part_m;      // [rows, n_parts] largest logit of each part
  const float* part_s;      // [rows, n_parts] sums of exp(logit - part_m), or nullptr: row_lse is there
  const float* row_lse;     // [rows]
  const float* score;       // [rows]
  const int32_t* size;      // [rows]
  int32_t beams, picks, n_parts, n_base_parts;
  int32_t base_columns, hyper_columns, slot_shift;   // columns of a part; 1 << slot_shift: the larger of them
  int32_t V, cap, ld;
  int32_t* parent;          // [prompts, picks]
  int32_t* code;
  float* picked;
};

typedef unsigned long long Key;   // candidate (order-preserving image) << 32 | ~index: larger is better, equal ones by lower index; 0: none

__device__ __forceinline__ Key make_key(float cand, uint32_t index) {
  if (!(cand > kNegInf) || cand == INFINITY) return 0ull;      // (-inf: not to be picked; a NaN has no order)
  const uint32_t u = __float_as_uint(cand + 0.0f);             // (-0 counts as 0)
  return ((Key)((u & 0x80000000u) ? ~u : (u | 0x80000000u)) << 32) | (uint32_t)~index;
}

__device__ __forceinline__ float key_value(Key k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float((u & 0x80000000u) ? (u & 0x7FFFFFFFu) : ~u);
}

__device__ __forceinline__ Key max_key(Key a, Key b) { return a > b ? a : b; }

constexpr int P_THREADS = 1024, P_GROUPS = 256, P_LIST = 2048, P_KEPT = 4, P_PARTS = 8192;

struct PickLds {
  Key group[P_GROUPS];
  Key list[P_LIST];
  Key top[Z2Z_MAX_PICK];
  Key threshold;
  Key wave[P_THREADS / 64];
  uint32_t found;
};

// The n largest of key(0) .. key(count - 1), all different where they are not 0, in order into l.top; the rest of l.top is 0.
// The threads fall into 64 groups (n up to 16) or 256, each with the maximum of its keys; the n-th largest of those maxima is a bound that
// at least n keys reach and at most n groups' worth: they are listed and ranked against each other.  A list that does
// not fit (keys so arranged that many large ones fall to one group) is left for n passes, each taking the largest key below the last.
// Up to 4 keys a thread stay in registers from the first look to the second; more are worked out again.
// read(i) is the value behind key i, from memory and without a branch, so that several are on the way together; make(i, value) the key.
template <typename R, typename F>
__device__ __forceinline__ void top_keys(PickLds& l, int n, uint32_t count, R read, F make) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool kept = count <= (uint32_t)(P_KEPT * P_THREADS);
  auto key = [&](uint32_t i) -> Key { return make(i, read(i)); };
  Key mine_all[P_KEPT], best = 0ull;
  if (kept) {
    float x[P_KEPT];
#pragma unroll
    for (int u = 0; u < P_KEPT; ++u) x[u] = read(min((uint32_t)(tid + u * P_THREADS), count - 1u));
#pragma unroll
    for (int u = 0; u < P_KEPT; ++u) {
      const uint32_t i = (uint32_t)(tid + u * P_THREADS);
      mine_all[u] = i < count ? make(i, x[u]) : 0ull;
      best = max_key(best, mine_all[u]);
    }
  } else {
    for (uint32_t i = tid; i < count; i += P_THREADS) best = max_key(best, key(i));
  }
  best = max_key(best, __shfl_xor(best, 1));
  best = max_key(best, __shfl_xor(best, 2));
  const int groups = n <= 16 ? 64 : P_GROUPS;
  if (groups == 64) {
    best = max_key(best, __shfl_xor(best, 4));
    best = max_key(best, __shfl_xor(best, 8));
    if ((tid & 15) == 0) l.group[tid >> 4] = best;
  } else if ((tid & 3) == 0) {
    l.group[tid >> 2] = best;
  }
  if (tid < n) l.top[tid] = 0ull;
  if (tid == 0) {
    l.found = 0u;
    l.threshold = 1ull;                  // fewer than n groups have any: all of theirs
  }
  __syncthreads();
  if (tid < groups) {
    const Key mine = l.group[tid];
    int above = 0;
#pragma unroll 8
    for (int i = 0; i < groups; ++i) above += l.group[i] > mine;
    if (above == n - 1 && mine != 0ull) l.threshold = mine;
  }
  __syncthreads();
  const Key threshold = l.threshold;
  auto append = [&](Key k) {
    if (k < threshold) return;
    const uint32_t at = atomicAdd(&l.found, 1u);
    if (at < (uint32_t)P_LIST) l.list[at] = k;
  };
  if (kept) {
#pragma unroll
    for (int u = 0; u < P_KEPT; ++u) append(mine_all[u]);
  } else {
    for (uint32_t i = tid; i < count; i += P_THREADS) append(key(i));
  }
  __syncthreads();
  const uint32_t found = l.found;
  if (found <= (uint32_t)P_LIST) {
    for (uint32_t i = tid; i < found; i += P_THREADS) {
      const Key mine = l.list[i];
      uint32_t above = 0u;
      for (uint32_t j0 = 0; j0 < found; j0 += 8u) {  // (8 reads on the way at a time)
        Key other[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) other[u] = l.list[min(j0 + (uint32_t)u, found - 1u)];
#pragma unroll
        for (int u = 0; u < 8; ++u) above += j0 + (uint32_t)u < found && other[u] > mine;
      }
      if (above < (uint32_t)n) l.top[above] = mine;
    }
  } else {
    Key last = ~0ull;
    for (int j = 0; j < n; ++j) {
      Key k = 0ull;
      for (uint32_t i = tid; i < count; i += P_THREADS) {
        const Key x = key(i);
        if (x < last) k = max_key(k, x);
      }
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) k = max_key(k, __shfl_xor(k, off));
      if (lane == 0) l.wave[wave] = k;
      __syncthreads();
      k = l.wave[0];
      for (int w = 1; w < P_THREADS / 64; ++w) k = max_key(k, l.wave[w]);
      if (tid == 0) l.top[j] = k;
      last = k;
      __syncthreads();
      if (last == 0ull) break;           // (uniform)
    }
  }
  __syncthreads();
}

// One workgroup per prompt.  A column among the n best lies in one of the n parts whose largest candidates are best (each of
// those has a better one, or an equal one of a lower index, than any other part), so only their logits are read.
__global__ void __launch_bounds__(P_THREADS) beam_pick_kernel(PickArgs a) {
  __shared__ PickLds l;
  __shared__ int part_beam[Z2Z_MAX_PICK], part_from[Z2Z_MAX_PICK], part_end[Z2Z_MAX_PICK];
  __shared__ float lse[Z2Z_MAX_BEAMS], score[Z2Z_MAX_BEAMS];
  __shared__ int columns[Z2Z_MAX_BEAMS];
  __shared__ float best[P_PARTS];
  const int tid = threadIdx.x;
  const int row0 = blockIdx.x * a.beams;
  // (a prompt's parts stay at hand where they fit: their maxima serve the log-sum-exps and the choice of parts)
  const bool at_hand = a.part_s && a.beams * a.n_parts <= P_PARTS;
  if (tid < a.beams) {
    score[tid] = a.score[row0 + tid];
    columns[tid] = a.V + min(max(a.size[row0 + tid], 0), a.cap);
  }
  // the beams' log-sum-exps, given or merged from the parts here (a launch less): a wave per beam, 8 parts a lane on the way at a time
  if (a.part_s) {
    const int lane = tid & 63;
    for (int beam = tid >> 6; beam < a.beams; beam += P_THREADS / 64) {
      const float *pm = a.part_m + (size_t)(row0 + beam) * a.n_parts, *ps = a.part_s + (size_t)(row0 + beam) * a.n_parts;
      float m = kNegInf, sum = 0.f;
      for (int p0 = lane; p0 < a.n_parts; p0 += 8 * 64) {
        float x[8], y[8], top = kNegInf;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int p = p0 + 64 * u;
          x[u] = p < a.n_parts ? pm[p] : kNegInf;
          y[u] = p < a.n_parts ? ps[p] : 0.f;
          if (at_hand && p < a.n_parts) best[beam * a.n_parts + p] = x[u];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) top = fmaxf(top, x[u]);
        const float up = fmaxf(m, top);
        sum = m == kNegInf ? sum : sum * __expf(m - up);
        // (an empty part adds nothing; a row's NaN stays NaN: a part that holds one has a NaN sum)
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += x[u] == kNegInf ? y[u] : y[u] * __expf(x[u] - up);
        m = up;
      }
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) {
        const float om = __shfl_xor(m, off), os = __shfl_xor(sum, off), up = fmaxf(m, om);
        sum = (m == kNegInf ? sum : sum * __expf(m - up)) + (om == kNegInf ? os : os * __expf(om - up));
        m = up;
      }
      if (lane == 0) lse[beam] = m + logf(sum);
    }
  } else if (tid < a.beams) {
    lse[tid] = a.row_lse[row0 + tid];
  }
  __syncthreads();
  const uint32_t n_parts = (uint32_t)a.n_parts, slot = (1u << a.slot_shift) - 1u;
  const int n = a.picks;
  // first the parts, then their columns (one piece of code for both: a single workgroup waits for its instructions, too)
#pragma unroll 1
  for (int phase = 0; phase < 2; ++phase) {
    auto read = [&](uint32_t i) -> float {
      if (phase == 0) return at_hand ? best[i] : a.part_m[(size_t)row0 * n_parts + i];      // (uniform)
      const uint32_t j = i >> a.slot_shift;
      return a.logits[(size_t)(row0 + part_beam[j]) * a.ld + min(part_from[j] + (int)(i & slot), a.ld - 1)];
    };
    auto make = [&](uint32_t i, float x) -> Key {
      if (phase == 0) {
        const uint32_t beam = i / n_parts;
        return make_key((x - lse[beam]) + score[beam], i);
      }
      const uint32_t j = i >> a.slot_shift, beam = (uint32_t)part_beam[j];
      const int c = part_from[j] + (int)(i & slot);
      const Key k = make_key((x - lse[beam]) + score[beam], beam * (uint32_t)a.ld + (uint32_t)c);
      return c < part_end[j] ? k : 0ull;
    };
    top_keys(l, n, phase == 0 ? (uint32_t)a.beams * n_parts : (uint32_t)n << a.slot_shift, read, make);
    if (phase == 0 && tid < n) {
      const Key part = l.top[tid];
      const uint32_t at = ~(uint32_t)part, beam = part ? at / n_parts : 0u, p = part ? at - beam * n_parts : 0u;
      int c = 0, end = 0;                            // (no such part: no columns)
      if (part && (int)p < a.n_base_parts) {
        c = (int)p * a.base_columns;
        end = min(c + a.base_columns, a.V);
      } else if (part) {
        c = a.V + ((int)p - a.n_base_parts) * a.hyper_columns;
        end = min(c + a.hyper_columns, columns[beam]);
      }
      part_beam[tid] = (int)beam;
      part_from[tid] = c;
      part_end[tid] = end;
    }
    __syncthreads();
  }
  if (tid < n) {
    const Key k = l.top[tid];
    const size_t out = (size_t)blockIdx.x * n + tid;
    const uint32_t at = ~(uint32_t)k;
    a.parent[out] = k ? (int32_t)(at / (uint32_t)a.ld) : -1;
    a.code[out] = k ? (int32_t)(at % (uint32_t)a.ld) : -1;
    a.picked[out] = k ? key_value(k) : kNegInf;
  }
}

// Largest logits of 256 columns each, where the logits' kernel left none per part: a wave per part.
__global__ void __launch_bounds__(256) part_max_kernel(const float* logits, const int32_t* size, int rows, int n_parts, int n_base_parts, int V,
                                                       int cap, float* part_m) {
  const int lane = threadIdx.x & 63;
  const long long wid = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int r = (int)(wid / n_parts), p = (int)(wid % n_parts);
  if (r >= rows) return;
  const int c0 = p < n_base_parts ? p * 256 : V + (p - n_base_parts) * 256;
  const int end = p < n_base_parts ? V : V + min(max(size[r], 0), cap);
  const float* x = logits + (size_t)r * (V + cap);
  float m = kNegInf;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int c = c0 + j * 64 + lane;
    if (c < end) m = fmaxf(m, x[c]);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  if (lane == 0) part_m[(size_t)r * n_parts + p] = m;
}

// ---- the move of the codebooks --------------------------------------------------------------------------------------------------
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;

struct ReorderArgs {
  LzwState st;
  const int32_t* source;    // [B], within the prompt
  u32x4* W;                 // [B, cap, d] or nullptr
  int32_t B, beams, chunks;
  long long first_entry;    // wave 0's, of prompts x cap
  int32_t entry_blocks;     // blocks that move entries; then, in the last launch, those of the hash tables, then one of the counts
  int32_t table_blocks;
};

__device__ __forceinline__ int source_of(const ReorderArgs& a, int prompt, int k) {
  const int s = a.source[prompt * a.beams + k];
  return s >= 0 && s < a.beams ? s : k;              // (no such beam: the slot keeps what it has)
}

// In place, whatever goes where: a thread that moves something has read all beams' values at its place before it writes
// the first, and no other thread touches that place.  N: beams, at most.
//   entries   a wave per prompt and entry: the lanes below N compare a beam's entry with its source's, the cache rows of those
//             that differ are moved 16 bytes a lane, then tokens and lengths
//   tables    a thread per prompt and bucket of 16 bytes
//   counts    a thread per prompt
// Bound by HBM: the cache rows of entries that differ, read and written once.
template <int N>
__global__ void __launch_bounds__(256) reorder_kernel(ReorderArgs a) {
  const int prompts = a.B / a.beams;
  if ((int)blockIdx.x < a.entry_blocks) {
    const int lane = threadIdx.x & 63;
    const long long wid = a.first_entry + (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int prompt = (int)(wid / a.st.cap), e = (int)(wid % a.st.cap);
    if (prompt >= prompts) return;
    const int b0 = prompt * a.beams, M = a.st.M;
    const bool on = lane < a.beams;
    const int k = on ? lane : 0;
    const int s = source_of(a, prompt, k);
    const size_t from = (size_t)(b0 + s) * a.st.cap + e, to = (size_t)(b0 + k) * a.st.cap + e;
    const int len = a.st.ent_len[from], old = a.st.ent_len[to];
    int32_t tok[Z2Z_MAX_M];
    bool differs = len != old;
#pragma unroll
    for (int j = 0; j < Z2Z_MAX_M; ++j)
      if (j < M) {
        tok[j] = a.st.ent_tokens[from * M + j];
        differs |= tok[j] != a.st.ent_tokens[to * M + j];
      }
    differs = differs && on && s != k;
    const uint32_t moved = (uint32_t)__ballot(differs), rows = (uint32_t)__ballot(differs && len > 0);
    if (moved == 0u) return;
    if (a.W && rows) {
      for (int c = lane; c < a.chunks; c += 64) {
        u32x4 x[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
          if ((rows >> i) & 1u) x[i] = a.W[((size_t)(b0 + __builtin_amdgcn_readlane(s, i)) * a.st.cap + e) * a.chunks + c];
#pragma unroll
        for (int i = 0; i < N; ++i)
          if ((rows >> i) & 1u) a.W[((size_t)(b0 + i) * a.st.cap + e) * a.chunks + c] = x[i];
      }
    }
    if (differs) {
      a.st.ent_len[to] = len;
#pragma unroll
      for (int j = 0; j < Z2Z_MAX_M; ++j)
        if (j < M) a.st.ent_tokens[to * M + j] = tok[j];
    }
    return;
  }
  if ((int)blockIdx.x < a.entry_blocks + a.table_blocks) {
    const int pairs = a.st.nslots >> 1;
    const long long at = (long long)((int)blockIdx.x - a.entry_blocks) * 256 + threadIdx.x;
    const int prompt = (int)(at / pairs), i = (int)(at % pairs);
    if (prompt >= prompts) return;
    u32x4* table = reinterpret_cast<u32x4*>(a.st.slots) + (size_t)prompt * a.beams * pairs + i;
    u32x4 x[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < a.beams) x[k] = table[(size_t)source_of(a, prompt, k) * pairs];
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < a.beams && source_of(a, prompt, k) != k) table[(size_t)k * pairs] = x[k];
    return;
  }
  for (int prompt = threadIdx.x; prompt < prompts; prompt += 256) {
    const int b0 = prompt * a.beams;
    int32_t size[N], code[N], len[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < a.beams) {
        const int b = b0 + source_of(a, prompt, k);
        size[k] = a.st.size[b];
        code[k] = a.st.prev_code[b];
        len[k] = a.st.prev_len[b];
      }
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < a.beams) {
        a.st.size[b0 + k] = size[k];
        a.st.prev_code[b0 + k] = code[k];
        a.st.prev_len[b0 + k] = len[k];
      }
  }
}

}  // namespace

int z2z_launch_beam_pick(z2z_ctx* c, const float* logits, const float* part_m, const float* part_s, int n_parts, int base_columns,
                         int hyper_columns, const float* row_lse, int beams, const float* score, int picks, int32_t* parent, int32_t* code, float* picked,
                         hipStream_t s) {
  PickArgs a;
  memset(&a, 0, sizeof(a));
  a.logits = logits;
  a.part_m = part_m;
  a.part_s = part_s;
  a.row_lse = row_lse;
  a.score = score;
  a.size = c->st.size;
  a.beams = beams;
  a.picks = picks;
  a.n_parts = n_parts;
  a.n_base_parts = (c->cfg.V + base_columns - 1) / base_columns;
  a.base_columns = base_columns;
  a.hyper_columns = hyper_columns;
  while ((1 << a.slot_shift) < std::max(base_columns, hyper_columns)) ++a.slot_shift;
  a.V = c->cfg.V;
  a.cap = c->cfg.cap;
  a.ld = c->cfg.V + c->cfg.cap;
  a.parent = parent;
  a.code = code;
  a.picked = picked;
  hipLaunchKernelGGL(beam_pick_kernel, dim3((unsigned)(c->cfg.B / beams)), dim3(P_THREADS), 0, s, a);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

int z2z_launch_part_max(z2z_ctx* c, const float* logits, float* part_m, int* n_parts, hipStream_t s) {
  const int n_base = (c->cfg.V + 255) / 256;
  *n_parts = n_base + (c->cfg.cap + 255) / 256;
  const long long waves = (long long)c->cfg.B * *n_parts;
  hipLaunchKernelGGL(part_max_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, logits, c->st.size, c->cfg.B, *n_parts, n_base,
                     c->cfg.V, c->cfg.cap, part_m);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

int z2z_launch_codebook_reorder(z2z_ctx* c, int32_t beams, const int32_t* source, void* W_hyper, hipStream_t s) {
  c->enc_kept = false;   // the rows a keeping encoder pass left behind belong to the codebook as it was
  ReorderArgs a;
  memset(&a, 0, sizeof(a));
  a.st = c->st;
  a.source = source;
  a.W = reinterpret_cast<u32x4*>(W_hyper);
  a.B = c->cfg.B;
  a.beams = beams;
  a.chunks = c->cfg.d / (c->cfg.dtype == Z2Z_BF16 ? 8 : 4);
  const long long prompts = a.B / beams, entries = prompts * c->cfg.cap, table_blocks = (prompts * (c->st.nslots >> 1) + 255) / 256;
  const long long most = kLaunchThreads / 256 - 1;                // blocks of a launch
  if (table_blocks >= most) return Z2Z_EUNSUPPORTED;
  // (one launch for up to 2^26 entries and tables; else entries ahead of it)
  auto launch = [&](long long entry_blocks, bool last) {
    a.entry_blocks = (int)entry_blocks;
    a.table_blocks = last ? (int)table_blocks : 0;
    const dim3 grid((unsigned)(entry_blocks + (last ? table_blocks + 1 : 0))), block(256);
    if (beams <= 4)
      hipLaunchKernelGGL(reorder_kernel<4>, grid, block, 0, s, a);
    else if (beams <= 8)
      hipLaunchKernelGGL(reorder_kernel<8>, grid, block, 0, s, a);
    else if (beams <= 16)
      hipLaunchKernelGGL(reorder_kernel<16>, grid, block, 0, s, a);
    else
      hipLaunchKernelGGL(reorder_kernel<32>, grid, block, 0, s, a);
    a.first_entry += entry_blocks * 4;
  };
  while ((entries - a.first_entry + 3) / 4 + table_blocks > most) launch(std::min((entries - a.first_entry + 3) / 4, most), false);
  launch((entries - a.first_entry + 3) / 4, true);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}
