// The common norm of a training step's gradients, and their clipping by it (gfx950): norm = sqrt(sum of all squares), out = min(1, max_norm / norm) * gradient.
//
// Bound by memory: every gradient is read once for the norm, then, where the norm is over max_norm or the output is another buffer, once more and written.  Two
// launches for up to 96 tensors: their list goes along as kernel arguments (nothing is copied to the device, and a captured call keeps its list).  The tensors are cut
// into chunks of 32 KiB, dealt out to workgroups in a fixed order, each of which leaves one sum in 64 bits; every workgroup of the second launch
// adds those up in the same order.  No atomics: the same inputs give the same bits.
#include "logits_common.h"

#include <algorithm>
#include <new>

namespace {

using z2z_logits::load_if;
using z2z_logits::pack_bf16;

constexpr int C_THREADS = 256;
constexpr int C_LOADS = 8;                                    // 16-byte loads a thread has in flight
constexpr int C_CHUNK = 16 * C_LOADS * C_THREADS;             // bytes
constexpr int C_LIST = 96;                                    // tensors of a launch

struct ClipList {
  const unsigned char* data[C_LIST];
  unsigned char* out[C_LIST];
  int64_t n[C_LIST];
  int32_t chunk0[C_LIST + 1];                                 // of every tensor, the first of its chunks
  uint8_t bf16[C_LIST];
  int32_t tensors;
};
static_assert(sizeof(ClipList) <= 3800, "kernel arguments are 4 KiB at most");

// Bytes ahead of the first 16-byte boundary; chunks are cut from there on, and the first takes these along.
__host__ __device__ __forceinline__ int head_bytes(const void* p) { return (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15); }

__device__ __forceinline__ int tensor_of(const ClipList& l, int chunk) {
  int lo = 0, hi = l.tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (l.chunk0[mid] <= chunk)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ float element(const unsigned char* p, int64_t i, bool bf16) {
  return bf16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << 16) : reinterpret_cast<const float*>(p)[i];
}

// The values of 16 bytes: eight bf16 or four floats.
template <bool BF16>
__device__ __forceinline__ void values_of(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (BF16) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    } else {
      x[i] = __uint_as_float(w[i]);
    }
  }
}

// The squares of 16 bytes, added to four chains.
template <bool BF16>
__device__ __forceinline__ void add_squares(const uint4& v, float4& s) {
  float x[8];
  values_of<BF16>(v, x);
  s = float4{fmaf(x[0], x[0], s.x), fmaf(x[1], x[1], s.y), fmaf(x[2], x[2], s.z), fmaf(x[3], x[3], s.w)};
  if (BF16) s = float4{fmaf(x[4], x[4], s.x), fmaf(x[5], x[5], s.y), fmaf(x[6], x[6], s.z), fmaf(x[7], x[7], s.w)};
}

// The 16-byte pieces of a chunk that belong to this thread; what does not exist reads as zeros.  begin: the tensor's first boundary; end: the last.
struct Span {
  const unsigned char* p;        // first piece of the chunk
  int pieces;                    // of this chunk
};
__device__ __forceinline__ Span span_of(const ClipList& l, int t, int chunk, int64_t* first) {
  const int size = l.bf16[t] ? 2 : 4;
  const int64_t bytes = l.n[t] * size, head = min((int64_t)head_bytes(l.data[t]), bytes);
  const int64_t whole = (bytes - head) >> 4, at = (int64_t)(chunk - l.chunk0[t]) * (C_CHUNK / 16);
  *first = head + at * 16;       // byte of the tensor at which the chunk's pieces start
  return Span{l.data[t] + *first, (int)max((int64_t)0, min((int64_t)(C_CHUNK / 16), whole - at))};
}

// The elements ahead of the first boundary and behind the last one: at most 7 and 7, of the first chunk's workgroup.  Element i of them, or -1.
__device__ __forceinline__ int64_t loose_element(const ClipList& l, int t, int i) {
  const int size = l.bf16[t] ? 2 : 4;
  const int64_t bytes = l.n[t] * size, head = min((int64_t)head_bytes(l.data[t]), bytes), tail = head + ((bytes - head) >> 4 << 4);
  const int n_head = (int)(head / size), n_tail = (int)((bytes - tail) / size);
  return i < n_head ? i : i - n_head < n_tail ? tail / size + (i - n_head) : -1;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ double workgroup_sum(double v, double* xch) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) xch[threadIdx.x >> 6] = v;
  __syncthreads();
  return (xch[0] + xch[1]) + (xch[2] + xch[3]);
}

__global__ void __launch_bounds__(C_THREADS) clip_squares_kernel(ClipList l, double* part) {
  __shared__ double xch[4];
  const int chunks = l.chunk0[l.tensors];
  double sum = 0.0;
  for (int chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
    const int t = tensor_of(l, chunk);
    const bool bf16 = l.bf16[t] != 0;
    int64_t first;
    const Span s = span_of(l, t, chunk, &first);
    uint4 v[C_LOADS];
#pragma unroll
    for (int i = 0; i < C_LOADS; ++i) {
      const int at = i * C_THREADS + (int)threadIdx.x;
      v[i] = load_if(at < s.pieces, reinterpret_cast<const uint4*>(s.p) + at);
    }
    float4 s4 = {0.f, 0.f, 0.f, 0.f};
    if (bf16) {
#pragma unroll
      for (int i = 0; i < C_LOADS; ++i) add_squares<true>(v[i], s4);
    } else {
#pragma unroll
      for (int i = 0; i < C_LOADS; ++i) add_squares<false>(v[i], s4);
    }
    const float squares = (s4.x + s4.y) + (s4.z + s4.w);
    uint32_t any = 0;                // (zeros are common: rows of an embedding that no token names)
#pragma unroll
    for (int i = 0; i < C_LOADS; ++i) any |= v[i].x | v[i].y | v[i].z | v[i].w;
    if ((squares > 1e-25f && squares < 1e37f) || any == 0) {
      sum += (double)squares;
    } else {
      // (out of the range in which squares keep their digits -- values beyond 1e18, or none above 1e-13: read again, and summed in 64 bits)
      for (int at = threadIdx.x; at < s.pieces; at += C_THREADS) {
        const int64_t e0 = (first + (int64_t)at * 16) / (bf16 ? 2 : 4);
        for (int i = 0; i < (bf16 ? 8 : 4); ++i) {
          const double x = (double)element(l.data[t], e0 + i, bf16);
          sum = fma(x, x, sum);
        }
      }
    }
    if (chunk == l.chunk0[t] && threadIdx.x < 16) {
      const int64_t e = loose_element(l, t, (int)threadIdx.x);
      const double x = e >= 0 ? (double)element(l.data[t], e, bf16) : 0.0;
      sum = fma(x, x, sum);
    }
  }
  sum = workgroup_sum(sum, xch);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The coefficient in two factors, power * rest: 1 and itself, or, where floats that small have few bits or none, 2^-100 and what is left.
struct Coefficient {
  float power, rest;
};
__device__ __forceinline__ float operator*(float x, const Coefficient& c) { return x * c.power * c.rest; }

template <bool BF16>
__device__ __forceinline__ uint4 scaled(const uint4& v, const Coefficient& c) {
  float x[8];
  values_of<BF16>(v, x);
#pragma unroll
  for (int i = 0; i < (BF16 ? 8 : 4); ++i) x[i] = x[i] * c;
  if (BF16) return uint4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
  return uint4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}

__device__ __forceinline__ void put(unsigned char* out, int64_t i, bool bf16, float x) {
  if (bf16)
    reinterpret_cast<uint16_t*>(out)[i] = (uint16_t)(pack_bf16(x, x) & 0xFFFFu);
  else
    reinterpret_cast<float*>(out)[i] = x;
}

// The chunks go from the last one back: what the first launch read last is in the caches still.
__global__ void __launch_bounds__(C_THREADS) clip_scale_kernel(ClipList l, const double* part, int parts, float max_norm, float* norm) {
  __shared__ double xch[4];
  double sum = 0.0;
  for (int i = threadIdx.x; i < parts; i += C_THREADS) sum += part[i];
  const double total = sqrt(workgroup_sum(sum, xch));
  // (a norm that is no finite number says nothing: the gradients stay as they are, for the caller to drop)
  const double ratio = total > (double)max_norm && total < 1.7e308 ? (double)max_norm / total : 1.0;
  const float c = (float)ratio;
  const Coefficient by = ratio < 0x1p-100 ? Coefficient{0x1p-100f, (float)(ratio * 0x1p100)} : Coefficient{1.0f, c};
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) {
    norm[0] = (float)total;
    norm[1] = c;
  }
  const int chunks = l.chunk0[l.tensors];
  for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
    const int chunk = chunks - 1 - k, t = tensor_of(l, chunk);
    const bool bf16 = l.bf16[t] != 0;
    unsigned char* out = l.out[t];
    if (c == 1.0f && out == l.data[t]) continue;
    int64_t first;
    const Span s = span_of(l, t, chunk, &first);
    const bool wide = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(l.data[t])) & 15) == 0;
    uint4 v[C_LOADS];
#pragma unroll
    for (int i = 0; i < C_LOADS; ++i) {
      const int at = i * C_THREADS + (int)threadIdx.x;
      v[i] = load_if(at < s.pieces, reinterpret_cast<const uint4*>(s.p) + at);
    }
#pragma unroll
    for (int i = 0; i < C_LOADS; ++i) {
      const int at = i * C_THREADS + (int)threadIdx.x;
      if (at >= s.pieces) continue;
      const uint4 y = c == 1.0f ? v[i] : bf16 ? scaled<true>(v[i], by) : scaled<false>(v[i], by);
      unsigned char* to = out + first + (int64_t)at * 16;
      if (wide) {
        // (past the caches, which hold what is still to be read: 0.8 GB in 36 tensors 457 -> 424 us, 4 GB 2218 -> 2180)
        typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
        __builtin_nontemporal_store(u32x4{y.x, y.y, y.z, y.w}, reinterpret_cast<u32x4*>(to));
      } else {                       // (on other boundaries than what is read)
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          if (bf16) {
            reinterpret_cast<uint16_t*>(to)[2 * h] = (uint16_t)w[h];
            reinterpret_cast<uint16_t*>(to)[2 * h + 1] = (uint16_t)(w[h] >> 16);
          } else {
            reinterpret_cast<uint32_t*>(to)[h] = w[h];
          }
        }
      }
    }
    if (chunk == l.chunk0[t] && threadIdx.x < 16) {
      const int64_t e = loose_element(l, t, (int)threadIdx.x);
      if (e >= 0) put(out, e, bf16, element(l.data[t], e, bf16) * by);
    }
  }
}

// Many sums as one, ahead of many launches that would each add them up: one workgroup.
constexpr int C_PARTS = 4096;
__global__ void __launch_bounds__(C_THREADS) clip_total_kernel(const double* part, int parts, double* total) {
  __shared__ double xch[4];
  double sum = 0.0;
  for (int i = threadIdx.x; i < parts; i += C_THREADS) sum += part[i];
  sum = workgroup_sum(sum, xch);
  if (threadIdx.x == 0) *total = sum;
}

struct Interval {
  uintptr_t begin, end;
  bool written;
};

}  // namespace

int z2z_launch_clip_gradients(z2z_ctx* c, const z2z_gradient* g, int n, float max_norm, float* norm, hipStream_t s) {
  // (a list's chunks are counted in 32 bits: 64 TiB)
  long long all = 0;
  for (int i = 0; i < n; ++i) {
    if (g[i].n > (1LL << 44)) return Z2Z_EUNSUPPORTED;
    all += std::max(1LL, ((long long)g[i].n * 4 + C_CHUNK - 1) / C_CHUNK);
  }
  if (all > 0x7FFF0000LL) return Z2Z_EUNSUPPORTED;
  // what is written overlaps nothing else
  Interval* iv = new (std::nothrow) Interval[2 * (size_t)n + 1];
  if (!iv) return Z2Z_ENOMEM;
  int m = 0;
  for (int i = 0; i < n; ++i) {
    if (g[i].n == 0) continue;
    const uintptr_t bytes = (uintptr_t)g[i].n * (g[i].dtype == Z2Z_BF16 ? 2 : 4);
    const uintptr_t in = reinterpret_cast<uintptr_t>(g[i].data), out = reinterpret_cast<uintptr_t>(g[i].out);
    iv[m++] = Interval{in, in + bytes, in == out};
    if (out && out != in) iv[m++] = Interval{out, out + bytes, true};
  }
  iv[m++] = Interval{reinterpret_cast<uintptr_t>(norm), reinterpret_cast<uintptr_t>(norm) + 2 * sizeof(float), true};
  std::sort(iv, iv + m, [](const Interval& a, const Interval& b) { return a.begin < b.begin; });
  uintptr_t read_to = 0, written_to = 0;
  bool clash = false;
  for (int i = 0; i < m; ++i) {
    clash = clash || iv[i].begin < written_to || (iv[i].written && iv[i].begin < read_to);
    uintptr_t& to = iv[i].written ? written_to : read_to;
    to = std::max(to, iv[i].end);
  }
  delete[] iv;
  if (clash) return Z2Z_EINVAL;

  const int lists = std::max(1, (n + C_LIST - 1) / C_LIST), most = 4 * c->num_cu;
  int rc = z2z_work_reserve(c, &c->clip_ws, ((size_t)lists * most + 1) * sizeof(double), s);
  if (rc != Z2Z_OK) return rc;
  double* part = reinterpret_cast<double*>(c->clip_ws.p);
  int parts = 0;
  for (int pass = 0; pass < 2; ++pass) {
    if (pass == 1 && parts > C_PARTS) {
      hipLaunchKernelGGL(clip_total_kernel, dim3(1), dim3(C_THREADS), 0, s, part, parts, part + parts);
      part += parts;
      parts = 1;
    }
    for (int first = 0; first < std::max(n, 1); first += C_LIST) {
      ClipList l = {};
      long long chunks = 0;
      for (int i = first; i < std::min(n, first + C_LIST); ++i) {
        // (the second launch has nothing to do with a tensor that counts for the norm alone: 4 GiB of them: one workgroup went over their chunks, 37 ms instead of 0.7)
        if (g[i].n == 0 || (pass == 1 && !g[i].out)) continue;
        const int t = l.tensors++;
        l.data[t] = reinterpret_cast<const unsigned char*>(g[i].data);
        l.out[t] = reinterpret_cast<unsigned char*>(g[i].out);
        l.n[t] = g[i].n;
        l.bf16[t] = g[i].dtype == Z2Z_BF16;
        const long long bytes = (long long)g[i].n * (l.bf16[t] ? 2 : 4);
        chunks += std::max(1LL, (bytes + C_CHUNK - 1) / C_CHUNK);
        l.chunk0[t + 1] = (int32_t)chunks;
      }
      const unsigned grid = (unsigned)std::max(1LL, std::min(chunks, (long long)most));
      if (pass == 0) {
        hipLaunchKernelGGL(clip_squares_kernel, dim3(grid), dim3(C_THREADS), 0, s, l, part + parts);
        parts += (int)grid;
      } else if (l.tensors > 0 || first == 0) {
        hipLaunchKernelGGL(clip_scale_kernel, dim3(grid), dim3(C_THREADS), 0, s, l, part, parts, max_norm, first == 0 ? norm : nullptr);
      }
    }
  }
  Z2Z_HIP_TRY(hipGetLastError());
  return Z2Z_OK;
}
