// The input side of a model over the extended vocabulary (gfx950): the lookup of a batch of code streams in the joint
// table [E ; W_hyper[b]], and its gradient.
//
// Section 2.2 of the zip2zip paper embeds a compressed sequence through the base embeddings and the hyper-embeddings of
// the sequence's own codebook.  X[b, i, :] = scale * (c < V ? E[c, :] : W_hyper[b, c - V, :]), c = codes[b, i], is a gather;
// its transpose adds dX[b, i, :] to the row that position named.
#include "hyper_embed_common.h"
#include "listed_rows.h"

#include <string.h>

#include <algorithm>

namespace {

using z2z_embed::u32x4;

constexpr uint32_t kNoKey = 0xFFFFFFFFu;
constexpr size_t kPastBytes = (size_t)128 << 20;     // half of the memory-side cache: what is written beyond that goes past it

struct LookupArgs {
  const int32_t* codes;     // [B, stride]
  const int32_t* n_codes;   // [B] or nullptr: stride
  const int32_t* size;      // [B] C_b
  int32_t B, V, cap, stride, chunks;   // chunks: 16-byte pieces of a row
  uint32_t sentinel;        // V + B * cap: what a position that names no row sorts by
};

__device__ __forceinline__ int codes_of(const LookupArgs& a, int b) {
  return a.n_codes ? min(max(a.n_codes[b], 0), a.stride) : a.stride;
}

__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t pack_two(float a, float b) {
  typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, z2z_embed::bf16x2));
}

// One 16-byte piece times scale: the product in fp32, rounded once to the storage type.
template <bool BF16>
__device__ __forceinline__ u32x4 scaled(u32x4 x, float scale) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    x[e] = BF16 ? pack_two(lo_bf16(x[e]) * scale, hi_bf16(x[e]) * scale) : __float_as_uint(__uint_as_float(x[e]) * scale);
  return x;
}

// Blocks [0, status_blocks): the status of sequence b, all of its codes looked over.  The others: a wave per position and `split`-th of its
// row, from number `first` on.  Bound by HBM: the rows written and each named row read once (popular ones come out of the caches).  PAST: the rows go out past the
// caches, where they are more than half of the memory-side one (8 x 4096 positions, three quarters in use, d = 4096, 0.2 GB written and 0.18 read at
// most: 65 -> 58 us with other rows before, 54 -> 48 over and over; the model finds fewer rows than that in the cache).
template <bool BF16, bool PAST>
__global__ void __launch_bounds__(256) embed_codes_kernel(LookupArgs a, const u32x4* E, const u32x4* W, u32x4* X, int32_t* status,
                                                          float scale, int split, int status_blocks, long long first) {
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x < status_blocks) {
    const int b = blockIdx.x, n = codes_of(a, b), columns = a.V + min(max(a.size[b], 0), a.cap);
    const int32_t* c = a.codes + (size_t)b * a.stride;
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += 256) bad |= c[i] < 0 || c[i] >= columns;
    const int any = __syncthreads_or(bad);
    if (threadIdx.x == 0) status[b] = any ? Z2Z_ST_BAD_CODE : Z2Z_ST_OK;
    return;
  }
  const long long wid = first + (long long)(blockIdx.x - (unsigned)status_blocks) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long pos = wid / split;
  const int part = (int)(wid % split);
  if (pos >= (long long)a.B * a.stride) return;
  const int b = (int)(pos / a.stride), i = (int)(pos % a.stride);
  if (i >= codes_of(a, b)) return;                   // rows behind a sequence's end stay as they were
  const int c = a.codes[pos];
  const bool base = c < a.V, named = c >= 0 && (base || c - a.V < min(max(a.size[b], 0), a.cap));
  const u32x4* row = base ? E + (size_t)(named ? c : 0) * a.chunks : W + ((size_t)b * a.cap + (named ? c - a.V : 0)) * a.chunks;
  u32x4* out = X + (size_t)pos * a.chunks;
  const u32x4 zero = {0u, 0u, 0u, 0u};
  constexpr int U = 4;
  for (int k0 = part * 64 + lane; k0 < a.chunks; k0 += U * 64 * split) {
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = named ? row[min(k0 + u * 64 * split, a.chunks - 1)] : zero;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + u * 64 * split < a.chunks) z2z_embed::store_chunk<PAST>(named ? scaled<BF16>(x[u], scale) : zero, out + k0 + u * 64 * split);
  }
}

// ---- gradient: positions sorted by the row they name -------------------------------------------------------------------------
// A row of the table collects the gradients of all its positions, in the order of the positions whatever the launch
// does: no float atomics.  The positions are sorted by their key -- the token, or V + b * cap + entry -- with a stable
// radix sort by digits of up to 10 bits, least significant first; equal keys then stand together in order of position.

constexpr int S_TILE = 4096;              // items of a workgroup: 16 waves, each up to 4 rounds of 64 in a row
constexpr int S_ROUNDS = S_TILE / 1024;
constexpr int S_DIGITS = 1024;

__device__ __forceinline__ uint32_t key_of(const LookupArgs& a, uint32_t i) {
  const uint32_t b = i / (uint32_t)a.stride, j = i - b * (uint32_t)a.stride;
  if ((int)j >= codes_of(a, (int)b)) return a.sentinel;
  const int c = a.codes[i];
  if (c < 0) return a.sentinel;
  if (c < a.V) return (uint32_t)c;
  return c - a.V < min(max(a.size[b], 0), a.cap) ? (uint32_t)a.V + b * (uint32_t)a.cap + (uint32_t)(c - a.V) : a.sentinel;
}

struct SortLds {
  uint16_t cnt[16][S_DIGITS];             // per wave: how often a digit came so far, then where its next one goes
  uint32_t wave_sum[16];
};

// Where every item of the tile goes among the tile's items: item (wave, round r, lane) is number wave * 64 * rounds + 64 r + lane.
// Equal digits within a wave's 64 are found by ballots, one per bit; the lanes below count.  Behind the last item of a
// tile stand dummies with all bits set: they stay behind every item, which are put in order before them.
// Returns per item its place, and leaves in l.cnt[0][d] the place of the tile's first item with digit d.
__device__ __forceinline__ void tile_places(SortLds& l, const uint32_t (&key)[S_ROUNDS], int rounds, int shift, int bits, uint32_t (&place)[S_ROUNDS]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t mask = (1u << bits) - 1u;
  const int digits = 1 << bits;
  for (int i = tid; i < 16 * S_DIGITS / 2; i += 1024) reinterpret_cast<uint32_t*>(l.cnt)[i] = 0u;
  __syncthreads();
  volatile uint16_t* mine = l.cnt[wave];
  uint32_t rank[S_ROUNDS];
#pragma unroll
  for (int r = 0; r < S_ROUNDS; ++r) {
    rank[r] = 0u;
    if (r < rounds) {                     // (uniform)
      const uint32_t digit = (key[r] >> shift) & mask;
      uint64_t peers = ~0ull;
      for (int k = 0; k < bits; ++k) {
        const bool bit = (digit >> k) & 1u;
        const uint64_t m = __ballot(bit);
        peers &= bit ? m : ~m;
      }
      const uint32_t before = mine[digit];
      const uint32_t below = (uint32_t)__popcll(peers & ((1ull << lane) - 1ull));
      __builtin_amdgcn_wave_barrier();    // (a wave's LDS operations are carried out in order: all read before one writes)
      if (below == 0u) mine[digit] = (uint16_t)(before + (uint32_t)__popcll(peers));
      __builtin_amdgcn_wave_barrier();
      rank[r] = before + below;
    }
  }
  __syncthreads();
  uint32_t total = 0u;
  uint16_t of_wave[16];
  if (tid < digits) {
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      of_wave[w] = (uint16_t)total;
      total += l.cnt[w][tid];
    }
  }
  uint32_t incl = total;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
  }
  if (lane == 63) l.wave_sum[wave] = incl;
  __syncthreads();
  uint32_t first = incl - total;
  for (int w = 0; w < wave; ++w) first += l.wave_sum[w];
  if (tid < digits) {
#pragma unroll
    for (int w = 0; w < 16; ++w) l.cnt[w][tid] = (uint16_t)(first + of_wave[w]);
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < S_ROUNDS; ++r)
    if (r < rounds) place[r] = (uint32_t)l.cnt[wave][(key[r] >> shift) & mask] + rank[r];
}

// A sort's launches are a few workgroups bound by latency; the others write zeros meanwhile: 16-byte pieces [begin, end) of the base gradient.
struct Zeros {
  u32x4* p;
  size_t begin, end;
  bool past;                // past the caches
};

// 16-byte pieces from, from + step .. below end.  (Two loops: of a choice within one the compiler makes a single plain store.)
__device__ __forceinline__ void store_zeros(u32x4* p, size_t from, size_t end, size_t step, bool past) {
  const u32x4 zero = {0u, 0u, 0u, 0u};
  if (past)
    for (size_t i = from; i < end; i += step) __builtin_nontemporal_store(zero, p + i);
  else
    for (size_t i = from; i < end; i += step) p[i] = zero;
}

__device__ __forceinline__ void write_zeros(const Zeros& z, uint32_t block, uint32_t blocks) {
  store_zeros(z.p, z.begin + (size_t)block * 1024 + threadIdx.x, z.end, (size_t)blocks * 1024, z.past);
}

// Up to S_TILE positions: the whole sort in one workgroup, from pass to pass through LDS.  (joins: join_kernel's counter, cleared here.)
// LISTED: the other workgroups add the listed rows of a teacher's gradient meanwhile (122 rows of 33, d = 1024: 14.2 us for both, 12.5 + 9.6 in a launch
// of their own behind).
template <bool LISTED>
__global__ void __launch_bounds__(1024) sort_small_kernel(LookupArgs a, uint32_t n, int bits, int passes, uint32_t* skey, uint32_t* spos,
                                                          uint32_t* joins, Zeros z, z2z_listed::ListedArgs listed) {
  __shared__ SortLds l;
  __shared__ uint32_t xkey[S_TILE];
  __shared__ uint16_t xpos[S_TILE];
  if (blockIdx.x > 0) {
    if (LISTED)
      z2z_listed::add_listed_rows(listed, (long long)(blockIdx.x - 1u) * 16 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    else
      write_zeros(z, blockIdx.x - 1u, gridDim.x - 1u);
    return;
  }
  if (joins && threadIdx.x == 0) *joins = 0u;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rounds = (int)((n + 1023u) / 1024u);
  uint32_t key[S_ROUNDS], pos[S_ROUNDS], place[S_ROUNDS];
#pragma unroll
  for (int r = 0; r < S_ROUNDS; ++r) {
    const uint32_t i = (uint32_t)(wave * 64 * rounds + 64 * r + lane);
    pos[r] = i;
    key[r] = r < rounds && i < n ? key_of(a, i) : kNoKey;
    place[r] = 0u;
  }
  for (int p = 0; p < passes; ++p) {
    tile_places(l, key, rounds, p * bits, bits, place);
#pragma unroll
    for (int r = 0; r < S_ROUNDS; ++r)
      if (r < rounds) {
        xkey[place[r]] = key[r];
        xpos[place[r]] = (uint16_t)pos[r];
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < S_ROUNDS; ++r)
      if (r < rounds) {
        const int i = wave * 64 * rounds + 64 * r + lane;
        key[r] = xkey[i];
        pos[r] = xpos[i];
      }
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < S_ROUNDS; ++r) {
    const uint32_t i = (uint32_t)(wave * 64 * rounds + 64 * r + lane);
    if (r < rounds && i < n) {
      skey[i] = key[r];
      spos[i] = pos[r];
    }
  }
}

// More: per pass, every tile counts its digits ...
__global__ void __launch_bounds__(1024) sort_count_kernel(LookupArgs a, uint32_t n, uint32_t tiles, const uint32_t* key_in, int shift, int bits,
                                                          uint32_t* count, uint32_t* joins, Zeros z) {
  __shared__ uint32_t cnt[S_DIGITS];
  const int digits = 1 << bits;
  if (blockIdx.x >= tiles) {
    write_zeros(z, blockIdx.x - tiles, gridDim.x - tiles);
    return;
  }
  if (joins && blockIdx.x == 0 && threadIdx.x == 0) *joins = 0u;
  for (int i = threadIdx.x; i < digits; i += 1024) cnt[i] = 0u;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < S_ROUNDS; ++r) {
    const uint32_t i = blockIdx.x * (uint32_t)S_TILE + 1024u * r + threadIdx.x;
    if (i < n) atomicAdd(&cnt[((key_in ? key_in[i] : key_of(a, i)) >> shift) & (uint32_t)(digits - 1)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < digits; i += 1024) count[(size_t)blockIdx.x * digits + i] = cnt[i];
}

// ... and puts its items behind those of smaller digits and of the same digit in the tiles before.
__global__ void __launch_bounds__(1024) sort_place_kernel(LookupArgs a, uint32_t n, uint32_t n_tiles, const uint32_t* key_in, const uint32_t* pos_in,
                                                          int shift, int bits, const uint32_t* count, uint32_t* key_out, uint32_t* pos_out,
                                                          Zeros z) {
  __shared__ SortLds l;
  __shared__ uint32_t go[S_DIGITS];       // where the tile's first item with the digit goes
  __shared__ uint32_t sums[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (blockIdx.x >= n_tiles) {
    write_zeros(z, blockIdx.x - n_tiles, gridDim.x - n_tiles);
    return;
  }
  const int digits = 1 << bits, tiles = (int)n_tiles;
  const uint32_t t0 = blockIdx.x * (uint32_t)S_TILE;
  uint32_t key[S_ROUNDS], pos[S_ROUNDS], place[S_ROUNDS];
#pragma unroll
  for (int r = 0; r < S_ROUNDS; ++r) {
    const uint32_t i = t0 + (uint32_t)(wave * 64 * S_ROUNDS + 64 * r + lane);
    const bool there = i < n;
    key[r] = there ? (key_in ? key_in[i] : key_of(a, i)) : kNoKey;
    pos[r] = there && pos_in ? pos_in[i] : i;
    place[r] = 0u;
  }
  uint32_t total = 0u, before = 0u;
  if (tid < digits)
    for (int t0 = 0; t0 < tiles; t0 += 8) {          // (eight loads on the way at a time)
      uint32_t x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = count[(size_t)min(t0 + u, tiles - 1) * digits + tid];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        total += t0 + u < tiles ? x[u] : 0u;
        before += t0 + u < (int)blockIdx.x ? x[u] : 0u;
      }
    }
  uint32_t incl = total;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
  }
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  uint32_t first = incl - total;
  for (int w = 0; w < wave; ++w) first += sums[w];
  if (tid < digits) go[tid] = first + before;
  tile_places(l, key, S_ROUNDS, shift, bits, place);       // (its barriers make `go` visible)
#pragma unroll
  for (int r = 0; r < S_ROUNDS; ++r) {
    const uint32_t i = t0 + (uint32_t)(wave * 64 * S_ROUNDS + 64 * r + lane);
    if (i < n) {
      const uint32_t digit = (key[r] >> shift) & (uint32_t)(digits - 1);
      const uint32_t to = go[digit] + (place[r] - (uint32_t)l.cnt[0][digit]);
      key_out[to] = key[r];
      pos_out[to] = pos[r];
    }
  }
}

// ---- gradient: sums over runs of equal keys -----------------------------------------------------------------------------------
// What is summed up, and where to (KIND):
//   LOOKUP_BF16, LOOKUP_F32   the rows of dX, a position's own each; base rows are fp32
//   WEIGHTED                  weight[position] times row position / per_row of a bf16 matrix; to sums, fp32 rows of their own: a table row's is
//                             slot[row] (the row itself, or where there are fewer positions than rows the number of its first sorted position)
enum { LOOKUP_BF16 = 0, LOOKUP_F32 = 1, WEIGHTED = 2 };

// Sorted positions of a wave: 8 where there are few, so that more waves share them, 32 or 64 else (sums that cross the ends of a piece go
// through memory, [pieces, d] twice, and a teacher's lists have K positions a row).
constexpr int kShortPiece = 8;
int long_piece(int kind) { return kind == WEIGHTED ? 64 : 32; }
// Positions from which on the pieces are long.
long long long_from(int kind, int slices) { return (4096LL * long_piece(kind) + slices - 1) / slices; }

struct GradArgs {
  const u32x4* dX;
  const float* weight;
  const uint32_t* skey;
  const uint32_t* spos;
  void* dE;
  void* dW;
  float* head;                            // [pieces, d]: the sum of a run that began in an earlier piece
  float* tail;                            // [pieces, d]: the sum of a run that begins here and goes on
  uint32_t* joins;                        // how many runs cross pieces, then the pieces that they begin in, in any order
  uint32_t n, pieces, piece, V, sentinel;
  uint32_t fill_from;                     // first row of the joint table that reduce_kernel looks after (those below are zeros already)
  int32_t chunks, slices, d, add, fill_blocks, per_row;
  bool past;                              // zeros past the caches
  float scale;
  float* sums;                            // WEIGHTED
  int32_t* slot;
  int32_t by_row;
};

// N consecutive features of a table row := (+=) scale * sum.  first: the sorted position that its run begins at (WEIGHTED).
template <int KIND, int N>
__device__ __forceinline__ void store_row(const GradArgs& a, uint32_t key, uint32_t first, size_t at, const float (&sum)[N]) {
  if (KIND == WEIGHTED) {
    float4* to = reinterpret_cast<float4*>(a.sums + (size_t)(a.by_row ? key : first) * a.d + at);
#pragma unroll
    for (int q = 0; q < N / 4; ++q) to[q] = float4{sum[4 * q], sum[4 * q + 1], sum[4 * q + 2], sum[4 * q + 3]};
    return;
  }
  float x[N];
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = sum[e] * a.scale;
  const size_t row = key < a.V ? (size_t)key * a.d : (size_t)(key - a.V) * a.d;
  if (KIND == LOOKUP_F32 || (KIND == LOOKUP_BF16 && key < a.V)) {
    float4* to = reinterpret_cast<float4*>(reinterpret_cast<float*>(key < a.V ? a.dE : a.dW) + row + at);
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      float4 o = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
      if (a.add) {
        const float4 was = to[q];
        o = float4{was.x + o.x, was.y + o.y, was.z + o.z, was.w + o.w};
      }
      to[q] = o;
    }
    return;
  }
  uint2* to = reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(key < a.V ? a.dE : a.dW) + row + at);
#pragma unroll
  for (int q = 0; q < N / 4; ++q) {
    if (a.add) {
      const uint2 was = to[q];
      x[4 * q] += lo_bf16(was.x);
      x[4 * q + 1] += hi_bf16(was.x);
      x[4 * q + 2] += lo_bf16(was.y);
      x[4 * q + 3] += hi_bf16(was.y);
    }
    to[q] = uint2{pack_two(x[4 * q], x[4 * q + 1]), pack_two(x[4 * q + 2], x[4 * q + 3])};
  }
}

// The first sorted position in [lo, hi) whose key is at least `key` (hi: none), for a whole wave: 64 samples a step, so that a few loads
// follow each other where halving takes twenty.
__device__ __forceinline__ uint32_t lower_bound(const uint32_t* skey, uint32_t lo, uint32_t hi, uint32_t key) {
  const uint32_t lane = threadIdx.x & 63;
  while (hi - lo > 64u) {
    const uint32_t step = (hi - lo + 63u) / 64u, at = lo + lane * step;
    const uint32_t smaller = (uint32_t)__popcll(__ballot(at < hi && skey[min(at, hi - 1u)] < key));
    if (smaller == 0u) return lo;
    hi = min(hi, lo + smaller * step);
    lo += (smaller - 1u) * step + 1u;
  }
  return lo + (uint32_t)__popcll(__ballot(lo + lane < hi && skey[min(lo + lane, hi - 1u)] < key));
}

// The first blocks: a wave per piece of sorted positions and 64 times 16 bytes of their rows, eight rows requested at a
// time, added in fp32 in order.  Runs inside the piece are stored, what crosses its ends is left for join_kernel.  The last fill_blocks
// write zeros to the table rows that no position names: a wave per 16 rows.
// Bound by HBM: dX read once, the gradients written once.  8 x 4096 positions of 24.6 k in use, V = 128256, d = 2048 (1.25 GB): zeros past the caches
// where the gradients are larger than half of the memory-side one 280 -> 240 us (128 MB of them, V = 32000, d = 1000 fp32: 31 -> 38), these blocks
// last 240 -> 237; row V - 1 in half of all positions 341 with its positions walked through by the wave that looks after it, 250 searched past.
template <int KIND, int PIECE>
__global__ void __launch_bounds__(256) reduce_kernel(GradArgs a) {
  const int lane = threadIdx.x & 63;
  constexpr bool BF16 = KIND != LOOKUP_F32;
  constexpr int EPC = BF16 ? 8 : 4;
  const uint32_t sum_blocks = gridDim.x - (uint32_t)a.fill_blocks;
  if (blockIdx.x >= sum_blocks) {
    const uint32_t first = a.fill_from + ((blockIdx.x - sum_blocks) * 4u + (threadIdx.x >> 6)) * 16u;
    uint32_t named = 0u;                             // a bit per row
    for (uint32_t at = lower_bound(a.skey, 0u, a.n, first); at < a.n;) {
      const uint32_t k = at + lane < a.n ? a.skey[at + lane] : kNoKey;
      const uint32_t row = k - first;
      uint32_t bits = k >= first && row < 16u ? 1u << row : 0u;
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) bits |= __shfl_xor(bits, off);
      named |= bits;
      const uint32_t last = (uint32_t)__builtin_amdgcn_readlane((int)k, 63);
      if (last - first >= 16u) break;
      at = lower_bound(a.skey, at + 64u, a.n, last + 1u);      // (a row that is named very often is left behind in a few steps)
    }
    for (int r = 0; r < 16; ++r) {
      if (((named >> r) & 1u) || first + (uint32_t)r >= a.sentinel) continue;
      const uint32_t k = first + (uint32_t)r;
      const int per_row = k < a.V ? a.d / 4 : a.chunks;
      u32x4* to = k < a.V ? reinterpret_cast<u32x4*>(a.dE) + (size_t)k * per_row : reinterpret_cast<u32x4*>(a.dW) + (size_t)(k - a.V) * per_row;
      store_zeros(to, (size_t)lane, (size_t)per_row, 64, a.past);
    }
    return;
  }
  const uint32_t wid = blockIdx.x * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t piece = wid / (uint32_t)a.slices;
  if (piece >= a.pieces) return;
  const int chunk = (int)(wid % (uint32_t)a.slices) * 64 + lane;
  const bool on = chunk < a.chunks;
  const uint32_t p0 = piece * PIECE;
  const int cnt = (int)min((uint32_t)PIECE, a.n - p0);
  const uint32_t my_key = lane < cnt ? a.skey[p0 + lane] : kNoKey;
  uint32_t my_pos = lane < cnt ? a.spos[p0 + lane] : 0u;
  float my_weight = 1.f;
  if (KIND == WEIGHTED) {
    my_weight = a.weight[my_pos];
    my_pos /= (uint32_t)a.per_row;
  }
  uint32_t key = __builtin_amdgcn_readfirstlane(my_key);
  if (key >= a.sentinel) return;
  uint32_t first = p0;
  const uint32_t prev = p0 > 0u ? a.skey[p0 - 1] : kNoKey, next = p0 + cnt < a.n ? a.skey[p0 + cnt] : kNoKey;
  bool began_before = prev == key;
  float acc[EPC];
#pragma unroll
  for (int e = 0; e < EPC; ++e) acc[e] = 0.f;
  const u32x4* column = a.dX + min(chunk, a.chunks - 1);
  for (int i0 = 0; i0 < PIECE; i0 += 8) {
    if (i0 >= cnt) break;
    u32x4 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = column[(size_t)(uint32_t)__builtin_amdgcn_readlane(my_pos, min(i0 + u, cnt - 1)) * a.chunks];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u;
      if (i >= cnt) break;
      if (key >= a.sentinel) return;                 // (positions that name nothing stand at the end)
      const float w = KIND == WEIGHTED ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(my_weight), i)) : 1.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (KIND == WEIGHTED) {
          acc[2 * e] = fmaf(w, lo_bf16(x[u][e]), acc[2 * e]);
          acc[2 * e + 1] = fmaf(w, hi_bf16(x[u][e]), acc[2 * e + 1]);
        } else if (BF16) {
          acc[2 * e] += lo_bf16(x[u][e]);
          acc[2 * e + 1] += hi_bf16(x[u][e]);
        } else {
          acc[e] += __uint_as_float(x[u][e]);
        }
      }
      const bool last = i + 1 == cnt;
      const uint32_t after = last ? next : (uint32_t)__builtin_amdgcn_readlane(my_key, min(i + 1, PIECE - 1));
      if (last || after != key) {
        const bool goes_on = last && after == key;
        if (goes_on && !began_before && chunk == 0) a.joins[1u + atomicAdd(a.joins, 1u)] = piece;
        if (KIND == WEIGHTED && !began_before && chunk == 0) a.slot[key] = (int32_t)(a.by_row ? key : first);
        if (on) {
          if (began_before || goes_on) {
            float4* to = reinterpret_cast<float4*>((began_before ? a.head : a.tail) + (size_t)piece * a.d + (size_t)chunk * EPC);
#pragma unroll
            for (int q = 0; q < EPC / 4; ++q) to[q] = float4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
          } else {
            store_row<KIND, EPC>(a, key, first, (size_t)chunk * EPC, acc);
          }
        }
#pragma unroll
        for (int e = 0; e < EPC; ++e) acc[e] = 0.f;
        began_before = false;
        key = after;
        first = p0 + (uint32_t)i + 1u;
      }
    }
  }
}

// Runs over several pieces, each 256 features at a time: the four waves of a block add a quarter of the run's pieces each, in order, and the quarters
// in order.
template <int KIND>
__global__ void __launch_bounds__(256) join_kernel(GradArgs a) {
  __shared__ float4 part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t groups = ((uint32_t)a.d + 255u) / 256u, jobs = a.joins[0] * groups;
  for (uint32_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    const uint32_t p = a.joins[1u + job / groups], p1 = (p + 1u) * a.piece;
    const uint32_t key = a.skey[p1];
    // the run's last piece: the last that begins with the key
    uint32_t q1 = p;
    for (;;) {
      const uint32_t q = q1 + 1u + (uint32_t)lane;
      const bool more = q < a.pieces && a.skey[min(q, a.pieces - 1u) * a.piece] == key;
      const uint32_t pieces = (uint32_t)__popcll(__ballot(more));
      q1 += pieces;
      if (pieces < 64u) break;
    }
    const int f = (int)(job % groups) * 256 + lane * 4;
    const bool on = f < a.d;
    const uint32_t heads = q1 - p, each = (heads + 3u) / 4u;
    const uint32_t from = p + 1u + min((uint32_t)wave * each, heads), to = p + 1u + min(((uint32_t)wave + 1u) * each, heads);
    float4 sum = {0.f, 0.f, 0.f, 0.f};
    if (on) {
      if (wave == 0) sum = *reinterpret_cast<const float4*>(a.tail + (size_t)p * a.d + f);
#pragma unroll 8
      for (uint32_t q = from; q < to; ++q) {
        const float4 x = *reinterpret_cast<const float4*>(a.head + (size_t)q * a.d + f);
        sum.x += x.x;
        sum.y += x.y;
        sum.z += x.z;
        sum.w += x.w;
      }
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && on) {
#pragma unroll
      for (int w = 1; w < 4; ++w) {
        const float4 x = part[w][lane];
        sum.x += x.x;
        sum.y += x.y;
        sum.z += x.z;
        sum.w += x.w;
      }
      const float s[4] = {sum.x, sum.y, sum.z, sum.w};
      store_row<KIND, 4>(a, key, KIND == WEIGHTED ? (uint32_t)a.slot[key] : 0u, (size_t)f, s);
    }
    __syncthreads();
  }
}

LookupArgs lookup_args(const z2z_ctx* c, const int32_t* codes, const int32_t* n_codes, int32_t stride) {
  LookupArgs a;
  a.codes = codes;
  a.n_codes = n_codes;
  a.size = c->st.size;
  a.B = c->cfg.B;
  a.V = c->cfg.V;
  a.cap = c->cfg.cap;
  a.stride = stride;
  a.chunks = c->cfg.d / (c->cfg.dtype == Z2Z_BF16 ? 8 : 4);
  a.sentinel = (uint32_t)((long long)c->cfg.V + (long long)c->cfg.B * c->cfg.cap);
  return a;
}

}  // namespace

int z2z_launch_embed_codes(z2z_ctx* c, const int32_t* codes, const int32_t* n_codes, int32_t stride, const void* E, const void* W_hyper,
                           float scale, void* X, int32_t* status, hipStream_t s) {
  const LookupArgs a = lookup_args(c, codes, n_codes, stride);
  const long long positions = (long long)a.B * stride;
  int split = 1;
  while (split < 16 && positions * split < 2048 && a.chunks > 64 * split) split *= 2;
  const dim3 block(256);
  const u32x4 *e = reinterpret_cast<const u32x4*>(E), *w = reinterpret_cast<const u32x4*>(W_hyper);
  u32x4* x = reinterpret_cast<u32x4*>(X);
  const bool past = (size_t)positions * a.chunks * 16 > kPastBytes;
  // (one launch for up to 2^26 positions, with the statuses; then more: kLaunchThreads)
  if (a.B >= kLaunchThreads / 256) return Z2Z_EUNSUPPORTED;
  const long long waves = positions * split;
  long long first = 0;
  int status_blocks = a.B;
  do {
    const long long most = (kLaunchThreads / 256 - status_blocks) * 4, n = std::min(waves - first, most);
    const dim3 grid((unsigned)(status_blocks + (n + 3) / 4));
    if (c->cfg.dtype == Z2Z_BF16 && past)
      hipLaunchKernelGGL((embed_codes_kernel<true, true>), grid, block, 0, s, a, e, w, x, status, scale, split, status_blocks, first);
    else if (c->cfg.dtype == Z2Z_BF16)
      hipLaunchKernelGGL((embed_codes_kernel<true, false>), grid, block, 0, s, a, e, w, x, status, scale, split, status_blocks, first);
    else if (past)
      hipLaunchKernelGGL((embed_codes_kernel<false, true>), grid, block, 0, s, a, e, w, x, status, scale, split, status_blocks, first);
    else
      hipLaunchKernelGGL((embed_codes_kernel<false, false>), grid, block, 0, s, a, e, w, x, status, scale, split, status_blocks, first);
    first += n;
    status_blocks = 0;
  } while (first < waves);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

namespace {

// Bytes of zeros that a sort's launch takes along at about its own length.
constexpr size_t kZerosSmall = (size_t)128 << 20, kZerosCount = (size_t)40 << 20, kZerosPlace = (size_t)96 << 20;

__global__ void __launch_bounds__(256) listed_rows_kernel(z2z_listed::ListedArgs a) {
  z2z_listed::add_listed_rows(a, (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
}

// How the work space of a sum by rows is laid out, and what its sort takes.  bytes: enough for every call of fewer positions, too, whose pieces may be
// short ones (d = 4096: 16383 positions of a lookup leave 64 MiB of sums, 32768 half of that), so that one call at the largest shape makes room for all.
struct SumPlan {
  uint32_t n, tiles, pieces;
  int bits, passes, piece;
  bool small;
  size_t o_key[2], o_pos[2], o_count, o_joins, o_head, o_tail, bytes;
};

bool plan_sum(const z2z_ctx* c, long long positions, int kind, SumPlan* p) {
  const int slices = (c->cfg.d / (kind == LOOKUP_F32 ? 4 : 8) + 63) / 64;
  const long long keys = (long long)c->cfg.V + (long long)c->cfg.B * c->cfg.cap;
  // (positions and rows of the joint table are 32-bit numbers here; reduce_kernel's blocks: 4 threads a row, 2 a position and slice)
  if (positions > 0x7FFFFFFFLL || keys > 0x7FFFFFFFLL || 4 * keys + 2 * positions * slices + (1LL << 27) > kLaunchThreads) return false;
  p->n = (uint32_t)positions;
  int key_bits = 1;
  while ((keys >> key_bits) != 0) ++key_bits;        // (the sentinel is a key, too)
  p->passes = (key_bits + 9) / 10;
  p->bits = (key_bits + p->passes - 1) / p->passes;
  p->tiles = (p->n + S_TILE - 1) / S_TILE;
  p->piece = positions < long_from(kind, slices) ? kShortPiece : long_piece(kind);
  p->pieces = (p->n + p->piece - 1) / p->piece;
  p->small = p->n <= (uint32_t)S_TILE;
  // sorted keys and positions (twice where the passes go through memory), the tiles' counts, sums that cross pieces
  p->bytes = 0;
  auto take = [&](size_t bytes) { const size_t at = p->bytes; p->bytes += (bytes + 255) / 256 * 256; return at; };
  for (int k = 0; k < 2; ++k) {
    p->o_key[k] = k == 0 || !p->small ? take((size_t)p->n * 4) : 0;
    p->o_pos[k] = k == 0 || !p->small ? take((size_t)p->n * 4) : 0;
  }
  p->o_count = p->small ? 0 : take((size_t)p->tiles * (1u << p->bits) * 4);
  p->o_joins = take(((size_t)p->pieces + 1) * 4);
  p->o_head = p->pieces > 1 ? take((size_t)p->pieces * c->cfg.d * 4) : 0;
  p->o_tail = p->pieces > 1 ? take((size_t)p->pieces * c->cfg.d * 4) : 0;
  SumPlan most;                                      // (of the calls with short pieces)
  if (p->piece != kShortPiece && plan_sum(c, long_from(kind, slices) - 1, kind, &most)) p->bytes = std::max(p->bytes, most.bytes);
  return true;
}

// Sort the positions, sum up the runs, join those that cross pieces.  g: what is summed and where to.
// listed (WEIGHTED): a teacher's listed rows for the hidden rows, in the sort's launch or in one of their own.
template <int KIND>
int launch_sum(const z2z_ctx* c, const LookupArgs& a, const SumPlan& p, unsigned char* ws, GradArgs g, hipStream_t s,
               const z2z_listed::ListedArgs& listed = z2z_listed::ListedArgs()) {
  auto words = [&](size_t at) { return reinterpret_cast<uint32_t*>(ws + at); };
  // zeros that go out with the sort: rows [0, fill_from) of the base gradient, `share` bytes a launch
  const size_t row16 = (size_t)c->cfg.d / 4;         // 16-byte pieces of a base row (fp32)
  g.past = (size_t)a.V * c->cfg.d * 4 + (size_t)a.B * a.cap * a.chunks * 16 > kPastBytes;
  Zeros z = {reinterpret_cast<u32x4*>(g.dE), 0, 0, g.past};
  unsigned fillers = 0;
  auto next_zeros = [&](size_t bytes) {
    z.begin = z.end;
    if (g.add) return;
    z.end = std::min(z.begin + bytes / 16 / row16 * row16, (size_t)a.V * row16);
    fillers = z.end > z.begin ? 512u : 0u;
  };
  uint32_t* joins = words(p.o_joins);
  int from = 0;
  if (p.n == 0u) {
    // (nothing to sort: zeros alone)
  } else if (p.small) {
    next_zeros(kZerosSmall);
    if (KIND == WEIGHTED) fillers = (unsigned)(((long long)listed.rows * listed.slices + 15) / 16);
    hipLaunchKernelGGL(sort_small_kernel<KIND == WEIGHTED>, dim3(1 + fillers), dim3(1024), 0, s, a, p.n, p.bits, p.passes, words(p.o_key[0]),
                       words(p.o_pos[0]), joins, z, listed);
  } else {
    if (KIND == WEIGHTED)
      hipLaunchKernelGGL(listed_rows_kernel, dim3((unsigned)(((long long)listed.rows * listed.slices + 3) / 4)), dim3(256), 0, s, listed);
    for (int k = 0; k < p.passes; ++k) {
      const uint32_t *key_in = k > 0 ? words(p.o_key[from]) : nullptr, *pos_in = k > 0 ? words(p.o_pos[from]) : nullptr;
      const int to = k > 0 ? from ^ 1 : 0;
      next_zeros(kZerosCount);
      hipLaunchKernelGGL(sort_count_kernel, dim3(p.tiles + fillers), dim3(1024), 0, s, a, p.n, p.tiles, key_in, k * p.bits, p.bits, words(p.o_count),
                         k == 0 ? joins : nullptr, z);
      next_zeros(kZerosPlace);
      hipLaunchKernelGGL(sort_place_kernel, dim3(p.tiles + fillers), dim3(1024), 0, s, a, p.n, p.tiles, key_in, pos_in, k * p.bits, p.bits,
                         words(p.o_count), words(p.o_key[to]), words(p.o_pos[to]), z);
      from = to;
    }
  }
  g.skey = p.n ? words(p.o_key[from]) : nullptr;
  g.spos = p.n ? words(p.o_pos[from]) : nullptr;
  g.head = p.pieces > 1 ? reinterpret_cast<float*>(ws + p.o_head) : nullptr;
  g.tail = p.pieces > 1 ? reinterpret_cast<float*>(ws + p.o_tail) : nullptr;
  g.n = p.n;
  g.pieces = p.pieces;
  g.piece = (uint32_t)p.piece;
  g.V = (uint32_t)a.V;
  g.sentinel = a.sentinel;
  g.chunks = a.chunks;
  g.slices = (a.chunks + 63) / 64;
  g.d = c->cfg.d;
  g.joins = joins;
  g.fill_from = (uint32_t)(z.end / row16);
  g.fill_blocks = g.add ? 0 : (int)(((long long)a.sentinel - g.fill_from + 63) / 64);
  const long long blocks = g.fill_blocks + ((long long)p.pieces * g.slices + 3) / 4;      // (plan_sum)
  if (p.piece == kShortPiece)
    hipLaunchKernelGGL((reduce_kernel<KIND, kShortPiece>), dim3((unsigned)blocks), dim3(256), 0, s, g);
  else
    hipLaunchKernelGGL((reduce_kernel<KIND, KIND == WEIGHTED ? 64 : 32>), dim3((unsigned)blocks), dim3(256), 0, s, g);
  // (8192 blocks at most: 2048 leave a teacher's lists, 524288 positions, at 92 us instead of 69)
  if (p.pieces > 1)
    hipLaunchKernelGGL(join_kernel<KIND>, dim3((unsigned)std::min<long long>((long long)p.pieces * ((c->cfg.d + 255) / 256), 8192)), dim3(256), 0, s, g);
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}

}  // namespace

int z2z_launch_embed_codes_backward(z2z_ctx* c, const int32_t* codes, const int32_t* n_codes, int32_t stride, float scale, const void* dX,
                                    int32_t flags, float* dE, void* dW_hyper, hipStream_t s) {
  const bool add = flags == Z2Z_GRAD_ADD;
  SumPlan p;
  if (!plan_sum(c, (long long)c->cfg.B * stride, c->cfg.dtype == Z2Z_BF16 ? LOOKUP_BF16 : LOOKUP_F32, &p)) return Z2Z_EUNSUPPORTED;
  if (p.n == 0u && add) return Z2Z_OK;
  const int rc = z2z_work_reserve(c, &c->lookup_ws, p.bytes, s);
  if (rc != Z2Z_OK) return rc;
  GradArgs g;
  memset(&g, 0, sizeof(g));
  g.dX = reinterpret_cast<const u32x4*>(dX);
  g.dE = dE;
  g.dW = dW_hyper;
  g.add = add ? 1 : 0;
  g.scale = scale;
  unsigned char* ws = reinterpret_cast<unsigned char*>(c->lookup_ws.p);
  const LookupArgs a = lookup_args(c, codes, n_codes, stride);
  return c->cfg.dtype == Z2Z_BF16 ? launch_sum<LOOKUP_BF16>(c, a, p, ws, g, s) : launch_sum<LOOKUP_F32>(c, a, p, ws, g, s);
}

namespace {

// A teacher's listed part of the gradient: the sum's own work space, then what it leaves to the products.
struct ListedPlan {
  SumPlan sum;
  size_t o_weight, o_grad, o_none, o_hidden, o_slot, o_sums, bytes;
  bool by_row;
};

bool plan_listed(const z2z_ctx* c, long long rows, int per_row, ListedPlan* p) {
  if (!plan_sum(c, rows * per_row, WEIGHTED, &p->sum) || rows * ((c->cfg.d + 511) / 512) * 64 + 1024 * 256 > kLaunchThreads) return false;
  const size_t n = p->sum.n, keys = (size_t)c->cfg.V + (size_t)c->cfg.B * c->cfg.cap, row = (size_t)c->cfg.d * sizeof(float);
  p->by_row = keys <= n;
  p->bytes = p->sum.bytes;
  auto take = [&](size_t bytes) { const size_t at = p->bytes; p->bytes += (bytes + 255) / 256 * 256; return at; };
  p->o_weight = take(n * sizeof(float));
  p->o_grad = take((size_t)rows * sizeof(float));
  p->o_none = take((size_t)rows * sizeof(int32_t));
  p->o_hidden = take((size_t)rows * row);
  p->o_slot = take(keys * sizeof(int32_t));
  p->o_sums = take((p->by_row ? keys : n) * row);
  return true;
}

}  // namespace

int z2z_listed_reserve(z2z_ctx* c, long long rows, int per_row, z2z_listed_part* l, hipStream_t s) {
  ListedPlan p;
  if (!plan_listed(c, rows, per_row, &p)) return Z2Z_EUNSUPPORTED;
  const int rc = z2z_work_reserve(c, &c->lookup_ws, p.bytes, s);
  if (rc != Z2Z_OK) return rc;
  unsigned char* ws = reinterpret_cast<unsigned char*>(c->lookup_ws.p);
  l->weight = reinterpret_cast<float*>(ws + p.o_weight);
  l->row_grad = reinterpret_cast<float*>(ws + p.o_grad);
  l->no_target = reinterpret_cast<int32_t*>(ws + p.o_none);
  l->hidden = reinterpret_cast<float*>(ws + p.o_hidden);
  l->slot = reinterpret_cast<int32_t*>(ws + p.o_slot);
  l->sums = reinterpret_cast<float*>(ws + p.o_sums);
  return Z2Z_OK;
}

int z2z_launch_listed(z2z_ctx* c, const int32_t* ids, long long rows, int per_row, const void* H, const void* W_base, const void* W_hyper,
                      const z2z_listed_part& part, hipStream_t s) {
  ListedPlan p;
  if (!plan_listed(c, rows, per_row, &p)) return Z2Z_EUNSUPPORTED;
  GradArgs g;
  memset(&g, 0, sizeof(g));
  g.dX = reinterpret_cast<const u32x4*>(H);
  g.weight = part.weight;
  g.add = 1;                                         // (rows that no position names are not looked after)
  g.per_row = per_row;
  g.sums = part.sums;
  g.slot = part.slot;
  g.by_row = p.by_row ? 1 : 0;
  const LookupArgs a = lookup_args(c, ids, nullptr, (int32_t)(rows / c->cfg.B * per_row));     // (a sequence's lists behind each other)
  z2z_listed::ListedArgs l;
  l.ids = ids;
  l.weight = part.weight;
  l.size = c->st.size;
  l.W_base = reinterpret_cast<const uint4*>(W_base);
  l.W_hyper = reinterpret_cast<const uint4*>(W_hyper);
  l.sum = reinterpret_cast<float4*>(part.hidden);
  l.rows = (int32_t)rows;
  l.rows_per_seq = (int32_t)(rows / c->cfg.B);
  l.V = c->cfg.V;
  l.cap = c->cfg.cap;
  l.K = per_row;
  l.n_chunks = a.chunks;
  l.slices = (a.chunks + 63) / 64;
  return launch_sum<WEIGHTED>(c, a, p.sum, reinterpret_cast<unsigned char*>(c->lookup_ws.p), g, s, l);
}
