// Clipping many gradients by their global norm:
//   norm = sqrt(sum over all tensors of g^2)   coef = min(1, max_norm / (norm + 1e-6))   dst = coef * src
// Two launches whatever the number of tensors.  Tensors are cut into chunks, which are listed in a table
// that the caller keeps on the device; a workgroup takes every G-th chunk, so the sums have one order.
// Squares and their sums are fp64, and so are norm and coef until they are rounded for the caller: the squares of fp32
// values leave fp32's range from 1.9e19 on (an exploding gradient, which is what clipping is for) and below 1e-23.
// Bound by memory: src is read twice, since nothing may be written before the whole norm is known.  The
// second launch goes through the chunks backwards: what was read last is in the 256 MB of the last cache,
// and it writes past that cache, so as not to push out what it has still to read (677 -> 642 us for 612
// million bf16 values; with 4096 workgroups instead of 2048, 635 us: 5.8 TB/s).
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>
#include <string.h>

#include <new>
#include <vector>

#include "../../include/dnb.h"

namespace {

constexpr int kThreads = 256;
constexpr int64_t kChunk = 16384;  // values
constexpr int kMost = 4096;        // workgroups

struct Chunk {
  const void* src;
  void* dst;
  int32_t count, flags;  // flags: 1 bf16, 2 not in 16-byte pieces
};

typedef unsigned u4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ double square_add(float v, double s) { return fma((double)v, (double)v, s); }

template <typename T>
__device__ __forceinline__ double square_sum(const Chunk& c) {
  constexpr int V = 16 / sizeof(T);
  const T* p = (const T*)c.src;
  double s = 0.0;
  int tail = 0;
  if (!(c.flags & 2)) {
    const int vecs = c.count / V;
#pragma unroll 8
    for (int i = threadIdx.x; i < vecs; i += kThreads) {
      const uint4 q = reinterpret_cast<const uint4*>(p)[i];
      T v[V];
      __builtin_memcpy(v, &q, 16);
#pragma unroll
      for (int j = 0; j < V; ++j) s = square_add((float)v[j], s);
    }
    tail = vecs * V;
  }
  for (int i = tail + threadIdx.x; i < c.count; i += kThreads) s = square_add((float)p[i], s);
  return s;
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const Chunk& c, float f, float f2) {
  constexpr int V = 16 / sizeof(T);
  const T* p = (const T*)c.src;
  T* y = (T*)c.dst;
  int tail = 0;
  if (!(c.flags & 2)) {
    const int vecs = c.count / V;
#pragma unroll 8
    for (int i = threadIdx.x; i < vecs; i += kThreads) {
      const uint4 q = reinterpret_cast<const uint4*>(p)[i];
      T v[V];
      __builtin_memcpy(v, &q, 16);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = (T)((float)v[j] * f * f2);
      uint4 o;
      __builtin_memcpy(&o, v, 16);
      __builtin_nontemporal_store(__builtin_bit_cast(u4, o), reinterpret_cast<u4*>(y) + i);
    }
    tail = vecs * V;
  }
  for (int i = tail + threadIdx.x; i < c.count; i += kThreads) y[i] = (T)((float)p[i] * f * f2);
}

// the sum of a value of every thread of the workgroup, in every thread
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[kThreads / 64];
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) s += red[i];
  return s;
}

__global__ __launch_bounds__(kThreads) void k_clip_squares(const Chunk* table, int chunks, double* part) {
  double s = 0.0;
  for (int i = blockIdx.x; i < chunks; i += gridDim.x) {
    const Chunk c = table[i];
    s += c.flags & 1 ? square_sum<__bf16>(c) : square_sum<float>(c);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads) void k_clip_scale(const Chunk* table, int chunks, const double* part, int parts, float max_norm,
                                                         float* norm) {
  int at = chunks - 1 - (int)blockIdx.x;
  Chunk k = {};
  if (at >= 0) k = table[at];  // on its way while the norm is made
  double s = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
  s = block_sum(s);
  const double n = sqrt(s), c = max_norm / (n + 1e-6);
  const float coef = (float)(c > 1.0 ? 1.0 : c);  // NaN stays
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    norm[0] = (float)n;
    norm[1] = coef;
  }
  // a coef that fp32 does not hold to its last bit is applied in two factors, the second a power of two
  const bool tiny = c < 0x1p-120;
  const float f = tiny ? (float)(c * 0x1p100) : coef, f2 = tiny ? 0x1p-100f : 1.f;
  while (at >= 0) {
    if (k.src == k.dst && f == 1.f) {  // in place and nothing to do
    } else if (k.flags & 1) scale_chunk<__bf16>(k, f, f2);
    else scale_chunk<float>(k, f, f2);
    at -= gridDim.x;
    if (at >= 0) k = table[at];
  }
}

}  // namespace

struct dnb_clip {
  std::vector<Chunk> table;
  int groups;
};

extern "C" {

int dnb_clip_create(const void* const* src, void* const* dst, const int64_t* counts, const int32_t* dtypes, int64_t tensors,
                    dnb_clip** out) {
  if (!out || (tensors > 0 && (!src || !dst || !counts || !dtypes))) return DNB_E_NULL;
  if (tensors < 0) return DNB_E_BADDESC;
  int64_t chunks = 0;
  for (int64_t i = 0; i < tensors; ++i) {
    if (counts[i] < 0 || (dtypes[i] != DNB_F32 && dtypes[i] != DNB_BF16)) return DNB_E_BADDESC;
    if (counts[i] > 0 && (!src[i] || !dst[i])) return DNB_E_NULL;
    const uintptr_t size = dtypes[i] == DNB_F32 ? 4 : 2;
    if (((uintptr_t)src[i] | (uintptr_t)dst[i]) & (size - 1)) return DNB_E_ALIGN;
    chunks += counts[i] / kChunk + (counts[i] % kChunk != 0);
    if (chunks > (1 << 26)) return DNB_E_RANGE;
  }
  dnb_clip* p = new (std::nothrow) dnb_clip();
  if (!p) return DNB_E_NOMEM;
  try {
    p->table.reserve((size_t)chunks);
  } catch (...) {
    delete p;
    return DNB_E_NOMEM;
  }
  for (int64_t i = 0; i < tensors; ++i) {
    const int64_t size = dtypes[i] == DNB_F32 ? 4 : 2;
    const bool odd = (((uintptr_t)src[i] | (uintptr_t)dst[i]) & 15) != 0;
    for (int64_t a = 0; a < counts[i]; a += kChunk)
      p->table.push_back({(const char*)src[i] + a * size, (char*)dst[i] + a * size,
                          (int32_t)(counts[i] - a < kChunk ? counts[i] - a : kChunk), (dtypes[i] == DNB_BF16 ? 1 : 0) | (odd ? 2 : 0)});
  }
  p->groups = chunks < 1 ? 1 : chunks < kMost ? (int)chunks : kMost;
  *out = p;
  return DNB_OK;
}

void dnb_clip_destroy(dnb_clip* plan) { delete plan; }

size_t dnb_clip_table_bytes(const dnb_clip* plan) { return plan ? plan->table.size() * sizeof(Chunk) : 0; }

int dnb_clip_table(const dnb_clip* plan, void* host) {
  if (!plan || (!host && !plan->table.empty())) return DNB_E_NULL;
  if (!plan->table.empty()) memcpy(host, plan->table.data(), plan->table.size() * sizeof(Chunk));
  return DNB_OK;
}

size_t dnb_clip_workspace_bytes(const dnb_clip* plan) { return plan ? (size_t)plan->groups * sizeof(double) : 0; }

int dnb_clip_run(const dnb_clip* plan, const void* table, float max_norm, float* norm, void* workspace, void* stream) {
  if (!plan || !norm || !workspace || (!table && !plan->table.empty())) return DNB_E_NULL;
  if (!(max_norm >= 0.f)) return DNB_E_BADDESC;
  if (((uintptr_t)table & 15) || ((uintptr_t)workspace & 15) || ((uintptr_t)norm & 3)) return DNB_E_ALIGN;
  hipStream_t st = (hipStream_t)stream;
  const int chunks = (int)plan->table.size();
  hipLaunchKernelGGL(k_clip_squares, dim3(plan->groups), dim3(kThreads), 0, st, (const Chunk*)table, chunks, (double*)workspace);
  if (hipGetLastError() != hipSuccess) return DNB_E_LAUNCH;
  hipLaunchKernelGGL(k_clip_scale, dim3(plan->groups), dim3(kThreads), 0, st, (const Chunk*)table, chunks, (const double*)workspace,
                     plan->groups, max_norm, norm);
  return hipGetLastError() == hipSuccess ? DNB_OK : DNB_E_LAUNCH;
}

}  // extern "C"
