// Rotary positions: each pair (a, b) of the first rotary_dim values of a head is turned by
// position * turn of the pair (in full turns) and scaled by `factor`:
//   a' = factor (a cos - b sin)      b' = factor (b cos + a sin)
// Bound by memory (16-byte pieces, every value read once and written once): 8191 rows of 24 heads of 128 in fp32
// in 40 us, 5.0 TB/s, as a copy.  The angles of a row are the
// same for all its heads: a workgroup computes them once for its rows into LDS.  position * turn is taken
// in 64 bits, of which only the fraction of a turn is kept: at position 131072 an fp32 product would be
// off by 1/64 of a radian.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "../../include/dnb.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxAngles = 1024;  // (row, pair) angles of a workgroup in LDS
constexpr unsigned kAcross = 1u << 22;  // workgroups along x, then z: less than 2^32 threads in one dimension

struct RopeArgs {
  const void* x;
  void* y;
  const int32_t* pos;
  const double* turns;
  int64_t rows, xs, ys;
  int heads, dim, half;     // half: pairs of a head
  int rpw, hpw;             // rows and heads of a workgroup
  int uph;                  // units of a head: half / V pairs of vectors (or vectors), then the rest
  uint32_t magic;           // j / uph = umulhi(j, magic)
  float factor, sign;
};

template <typename T, int V>
struct __attribute__((aligned(sizeof(T) * V))) Vec {
  T v[V];
};

template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kThreads) void k_rope(RopeArgs A) {
  __shared__ float2 cs[kMaxAngles];
  const int64_t r0 = ((int64_t)blockIdx.z * kAcross + blockIdx.x) * A.rpw;
  if (r0 >= A.rows) return;
  const int nr = (int)min((int64_t)A.rpw, A.rows - r0);
  const int h0 = blockIdx.y * A.hpw, nh = min(A.hpw, A.heads - h0);
  for (int i = threadIdx.x; i < nr * A.half; i += kThreads) {
    const int r = i / A.half, p = i - r * A.half;
    const double t = (double)A.pos[r0 + r] * A.turns[p];
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    cs[i] = make_float2(c * A.factor, s * A.factor * A.sign);
  }
  __syncthreads();
  constexpr int PU = HALF ? 2 * V : V;  // values that a unit turns
  const int turned = 2 * A.half / PU, per_row = nh * A.uph;
  using W = Vec<T, V>;
  for (int r = 0; r < nr; ++r) {
    const T* x = (const T*)A.x + (r0 + r) * A.xs + (int64_t)h0 * A.dim;
    T* y = (T*)A.y + (r0 + r) * A.ys + (int64_t)h0 * A.dim;
    const float2* a = cs + r * A.half;
    for (int j = threadIdx.x; j < per_row; j += kThreads) {
      const int h = A.uph == 1 ? j : (int)__umulhi((uint32_t)j, A.magic), u = j - h * A.uph;
      const int64_t at = (int64_t)h * A.dim;
      if (u >= turned) {  // not turned
        const int64_t e = at + 2 * A.half + (u - turned) * V;
        *reinterpret_cast<W*>(y + e) = *reinterpret_cast<const W*>(x + e);
      } else if (HALF) {
        const W p = *reinterpret_cast<const W*>(x + at + u * V), q = *reinterpret_cast<const W*>(x + at + A.half + u * V);
        W po, qo;
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float2 t = a[u * V + k];
          const float f = (float)p.v[k], g = (float)q.v[k];
          po.v[k] = (T)(f * t.x - g * t.y);
          qo.v[k] = (T)(g * t.x + f * t.y);
        }
        *reinterpret_cast<W*>(y + at + u * V) = po;
        *reinterpret_cast<W*>(y + at + A.half + u * V) = qo;
      } else {
        const W p = *reinterpret_cast<const W*>(x + at + u * V);
        W po;
#pragma unroll
        for (int k = 0; k + 1 < V; k += 2) {
          const float2 t = a[(u * V + k) / 2];
          const float f = (float)p.v[k], g = (float)p.v[k + 1];
          po.v[k] = (T)(f * t.x - g * t.y);
          po.v[k + 1] = (T)(g * t.x + f * t.y);
        }
        *reinterpret_cast<W*>(y + at + u * V) = po;
      }
    }
  }
}

template <typename T, int V>
hipError_t launch(RopeArgs A, bool half_order, hipStream_t st) {
  const int pu = half_order ? 2 * V : V;
  A.uph = 2 * A.half / pu + (A.dim - 2 * A.half) / V;
  A.magic = (uint32_t)((0x100000000ull + A.uph - 1) / A.uph);
  // About four units a thread, over whole rows if a row has fewer and over a part of the heads if it has
  // more; where that leaves compute units idle, one unit a thread.
  const int64_t per_row = (int64_t)A.heads * A.uph, units = A.rows * per_row;
  const int64_t want = units >= 4ll * kThreads * 1024 ? 4 * kThreads : kThreads;
  A.rpw = (int)min(max(want / per_row, (int64_t)1), (int64_t)max(1, kMaxAngles / A.half));
  A.hpw = (int)min(max(want / A.uph, (int64_t)1), (int64_t)A.heads);
  const int64_t across = (A.rows + A.rpw - 1) / A.rpw;
  const dim3 grid((unsigned)min(across, (int64_t)kAcross), (unsigned)((A.heads + A.hpw - 1) / A.hpw), (unsigned)((across + kAcross - 1) / kAcross));
  if (half_order) hipLaunchKernelGGL((k_rope<T, V, true>), grid, dim3(kThreads), 0, st, A);
  else hipLaunchKernelGGL((k_rope<T, (V < 2 ? 2 : V), false>), grid, dim3(kThreads), 0, st, A);
  return hipGetLastError();
}

// The widest vectors, up to 16 bytes, that rows, heads and pairs consist of wholly.
template <typename T>
hipError_t launch_any(const RopeArgs& A, bool half_order, hipStream_t st) {
  const int64_t all = (half_order ? A.half : 2 * A.half) | A.dim | A.xs | A.ys;
  if (sizeof(T) == 2 && all % 8 == 0) return launch<T, (sizeof(T) == 2 ? 8 : 4)>(A, half_order, st);
  if (all % 4 == 0) return launch<T, 4>(A, half_order, st);
  if (all % 2 == 0) return launch<T, 2>(A, half_order, st);
  return launch<T, 1>(A, half_order, st);
}

int rope(const void* x, const int32_t* positions, const double* turns, void* y, int64_t rows, int64_t heads, int64_t head_dim,
         int64_t rotary_dim, int order, float factor, int dtype, int64_t x_stride, int64_t y_stride, float sign, void* stream) {
  if (order != DNB_ROPE_HALF && order != DNB_ROPE_INTERLEAVED) return DNB_E_BADDESC;
  if (dtype != DNB_F32 && dtype != DNB_BF16) return DNB_E_BADDESC;
  if (rows < 0 || heads < 1 || head_dim < 2 || head_dim % 2 != 0 || rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > head_dim)
    return DNB_E_BADDESC;
  if (rows > 0x7fffffff || heads > 4096 || head_dim > 1024) return DNB_E_RANGE;
  if (x_stride == 0) x_stride = heads * head_dim;
  if (y_stride == 0) y_stride = heads * head_dim;
  if (x_stride < heads * head_dim || y_stride < heads * head_dim || x_stride % 2 != 0 || y_stride % 2 != 0) return DNB_E_RANGE;
  if (rows == 0) return DNB_OK;
  if (!x || !positions || !turns || !y) return DNB_E_NULL;
  if (((uintptr_t)x & 15) || ((uintptr_t)y & 15) || ((uintptr_t)turns & 7) || ((uintptr_t)positions & 3)) return DNB_E_ALIGN;
  const RopeArgs A{x, y, positions, turns, rows, x_stride, y_stride, (int)heads, (int)head_dim, (int)(rotary_dim / 2),
                   0, 0, 0, 0, factor, sign};
  const bool half_order = order == DNB_ROPE_HALF;
  const hipError_t e = dtype == DNB_BF16 ? launch_any<__bf16>(A, half_order, (hipStream_t)stream)
                                         : launch_any<float>(A, half_order, (hipStream_t)stream);
  return e == hipSuccess ? DNB_OK : DNB_E_LAUNCH;
}

}  // namespace

extern "C" {

int dnb_op_rope_forward(const void* x, const int32_t* positions, const double* turns, void* y, int64_t rows, int64_t heads,
                        int64_t head_dim, int64_t rotary_dim, int order, float factor, int dtype, int64_t x_stride,
                        int64_t y_stride, void* stream) {
  return rope(x, positions, turns, y, rows, heads, head_dim, rotary_dim, order, factor, dtype, x_stride, y_stride, 1.f, stream);
}

int dnb_op_rope_backward(const void* dy, const int32_t* positions, const double* turns, void* dx, int64_t rows, int64_t heads,
                         int64_t head_dim, int64_t rotary_dim, int order, float factor, int dtype, int64_t dy_stride,
                         int64_t dx_stride, void* stream) {
  return rope(dy, positions, turns, dx, rows, heads, head_dim, rotary_dim, order, factor, dtype, dy_stride, dx_stride, -1.f, stream);
}

}  // extern "C"
