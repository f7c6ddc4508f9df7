// The norms around a block (root-mean-square norms, no mean taken out), with the block's gate and the
// residual's scale, in one pass over the rows:
//   h_new = scale r + gate * (b / rms(b) * w_post)        y = h_new / rms(h_new) * w_pre
// and its gradients.  Bound by memory: a row lies in registers between its reductions, so every tensor is
// read once and written once; the weights stay in registers over the rows of a workgroup.  The statistics
// are not kept from the forward pass: the backward pass has the rows in registers anyway.
// The backward pass holds five rows and as many vectors: from width 4104 that leaves one wave a SIMD, and above
// 8192 (1024 threads, 128 registers each) 180 to 292 bytes a lane go to scratch.  128 MB a tensor in bf16, 256 MB
// in fp32, vector gate, backward: width 4096 5.2 and 5.0 TB/s; 4104 2.0 and 4.4; 8192 2.7 and 5.0; 8200 1.5 and 2.3; 16384
// 2.2 and 3.1.  Forward: 4.0 to 5.4 TB/s at all of them (bf16 4104: 3.6).
// 16381 rows of 4096 in bf16, backward: 152 us (5.3 TB/s) and 8 us for the sums over workgroups; 6272 rows of 2208 in
// fp32 with a full gate: 46 us forward, 79 us backward (5.6 TB/s).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "../../include/dnb.h"

namespace {

struct NormArgs {
  const void *b, *r, *gate, *h, *dh, *dy;
  const float *w_post, *w_pre;
  void *h_new, *y, *db, *dr, *dgate;
  float *dw_post, *dw_pre, *part;
  int64_t rows;
  int width;
  float scale, eps;
};

template <typename T>
__device__ __forceinline__ void load8(float (&v)[8], const T* p) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
// STREAM: past the caches.  The backward pass writes so: its outputs would push out what it has still to
// read of the forward's (a step of 6272 rows of 2208 fp32: 143 -> 130 us; the forward's outputs so: 136 us).
template <bool STREAM = false, typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  auto put = [](auto* q, auto x) {
    if (STREAM) __builtin_nontemporal_store(x, q);
    else *q = x;
  };
  if constexpr (sizeof(T) == 4) {
    put(reinterpret_cast<f4*>(p), (f4){v[0], v[1], v[2], v[3]});
    put(reinterpret_cast<f4*>(p) + 1, (f4){v[4], v[5], v[6], v[7]});
  } else {
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (__bf16)v[i];
    put(reinterpret_cast<bf16x8*>(p), y);
  }
}

// Sums of N values over the TPR threads of a row, in every one of them.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*red)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int o = 32; o; o >>= 1) v[n] += __shfl_xor(v[n], o);
  if constexpr (TPR > 64) {
    constexpr int WAVES = TPR / 64;
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) red[w][n] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) t += red[i][n];
      v[n] = t;
    }
  }
}

// A row is TPR threads (a wave, four or sixteen) with NV vectors of 8 values each.
template <typename T, int TPR, int NV, int GATE, bool POST>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_norm_forward(NormArgs A) {
  constexpr int RPW = TPR < 256 ? 256 / TPR : 1;
  __shared__ float red[2][2][16][1];  // a row's two sums, two rows in turn: between uses of one place lies the other row's barrier
  const int t = threadIdx.x % TPR;
  float wp[NV][8], w[NV][8], gv[NV][8];
  bool in[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8;
    in[i] = c < A.width;
#pragma unroll
    for (int j = 0; j < 8; ++j) { wp[i][j] = 1.f; w[i][j] = 0.f; gv[i][j] = 1.f; }
    if (in[i]) {
      if (POST) load8(wp[i], A.w_post + c);
      load8(w[i], A.w_pre + c);
      if (GATE == DNB_GATE_VECTOR) load8(gv[i], (const float*)A.gate + c);
    }
  }
  const float inv_w = 1.f / A.width;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR; row < A.rows; row += (int64_t)gridDim.x * RPW, turn ^= 1) {
    const int64_t at = row * A.width;
    float b[NV][8], h[NV][8], g[NV][8], s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) { b[i][j] = 0.f; h[i][j] = 0.f; g[i][j] = gv[i][j]; }
      if (in[i]) {
        load8(b[i], (const T*)A.b + at + c);
        load8(h[i], (const T*)A.r + at + c);
        if (GATE == DNB_GATE_FULL) load8(g[i], (const T*)A.gate + at + c);
      }
    }
    float ib = 1.f;
    if (POST) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] = fmaf(b[i][j], b[i][j], s[0]);
      row_sums<TPR, 1>(s, red[turn][0]);
      ib = 1.f / sqrtf(s[0] * inv_w + A.eps);
    }
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[i][j] = fmaf(g[i][j], b[i][j] * ib * wp[i][j], A.scale * h[i][j]);
        s[0] = fmaf(h[i][j], h[i][j], s[0]);
      }
    row_sums<TPR, 1>(s, red[turn][1]);
    const float ih = 1.f / sqrtf(s[0] * inv_w + A.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!in[i]) continue;
      const int c = (t + i * TPR) * 8;
      store8((T*)A.h_new + at + c, h[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] *= ih * w[i][j];
      store8((T*)A.y + at + c, h[i]);
    }
  }
}

// xb = b / rms(b), xh = h / rms(h), t = dy * w_pre:
//   dH = dh + (t - xh mean(t xh)) / rms(h)       dr = scale dH       dw_pre = sum over rows of dy xh
//   du = dH gate w_post     db = (du - xb mean(du xb)) / rms(b)      dw_post = sum of dH gate xb
//   dgate = dH xb w_post (a vector: its sum over rows)
// The means need two reductions a row: (b b, h h, t h) at once, then du b.  A vector gate leaves
// dw_post and dgate the same sum over the rows, of dH xb, times gate and times w_post.
// A workgroup's sums over its rows go to part[workgroup][2][width].
template <typename T, int TPR, int NV, int GATE, bool POST>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_norm_backward(NormArgs A) {
  constexpr int RPW = TPR < 256 ? 256 / TPR : 1;
  __shared__ float red3[2][16][3], red1[2][16][1];
  const int t = threadIdx.x % TPR;
  float wp[NV][8], w[NV][8], gv[NV][8], s0[NV][8], s1[NV][8];
  bool in[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8;
    in[i] = c < A.width;
#pragma unroll
    for (int j = 0; j < 8; ++j) { wp[i][j] = 1.f; w[i][j] = 0.f; gv[i][j] = 1.f; s0[i][j] = s1[i][j] = 0.f; }
    if (in[i]) {
      if (POST) load8(wp[i], A.w_post + c);
      load8(w[i], A.w_pre + c);
      if (GATE == DNB_GATE_VECTOR) load8(gv[i], (const float*)A.gate + c);
    }
  }
  const float inv_w = 1.f / A.width;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR; row < A.rows; row += (int64_t)gridDim.x * RPW, turn ^= 1) {
    const int64_t at = row * A.width;
    float b[NV][8], h[NV][8], dh[NV][8], dy[NV][8], g[NV][8], s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) { b[i][j] = h[i][j] = dh[i][j] = dy[i][j] = 0.f; g[i][j] = gv[i][j]; }
      if (in[i]) {
        load8(b[i], (const T*)A.b + at + c);
        load8(h[i], (const T*)A.h + at + c);
        load8(dh[i], (const T*)A.dh + at + c);
        load8(dy[i], (const T*)A.dy + at + c);
        if (GATE == DNB_GATE_FULL) load8(g[i], (const T*)A.gate + at + c);
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (POST) s[0] = fmaf(b[i][j], b[i][j], s[0]);
        s[1] = fmaf(h[i][j], h[i][j], s[1]);
        s[2] = fmaf(dy[i][j] * w[i][j], h[i][j], s[2]);
      }
    row_sums<TPR, 3>(s, red3[turn]);
    const float ib = POST ? 1.f / sqrtf(s[0] * inv_w + A.eps) : 1.f;
    const float ih = 1.f / sqrtf(s[1] * inv_w + A.eps);
    const float mean = s[2] * ih * inv_w;
    float d[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float xh = h[i][j] * ih;
        s0[i][j] = fmaf(dy[i][j], xh, s0[i][j]);
        dh[i][j] += ih * (dy[i][j] * w[i][j] - xh * mean);
        b[i][j] *= ib;
        const float dx = dh[i][j] * b[i][j];
        s1[i][j] = fmaf(GATE == DNB_GATE_FULL ? g[i][j] : 1.f, dx, s1[i][j]);
        h[i][j] = dx * wp[i][j];                     // the gate's gradient
        dy[i][j] = dh[i][j] * g[i][j] * wp[i][j];    // du
        if (POST) d[0] = fmaf(dy[i][j], b[i][j], d[0]);
      }
    if (POST) row_sums<TPR, 1>(d, red1[turn]);
    const float m = d[0] * inv_w;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!in[i]) continue;
      const int c = (t + i * TPR) * 8;
      if (GATE == DNB_GATE_FULL) store8<true>((T*)A.dgate + at + c, h[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (POST) dy[i][j] = ib * (dy[i][j] - b[i][j] * m);
        dh[i][j] *= A.scale;
      }
      store8<true>((T*)A.db + at + c, dy[i]);
      store8<true>((T*)A.dr + at + c, dh[i]);
    }
  }
  // part rows: (workgroup, row of it)
  float* p = A.part + ((int64_t)blockIdx.x * RPW + threadIdx.x / TPR) * 2 * A.width;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (!in[i]) continue;
    const int c = (t + i * TPR) * 8;
    store8(p + c, s0[i]);
    store8(p + A.width + c, s1[i]);
  }
}

// Columns of the partial sums, in a fixed order: 16 a workgroup (64 bytes of a row), 64 threads a column.
// With 64 columns and 16 threads each (128 workgroups at width 4096) 512 parts took 11 us.
template <int GATE, bool POST>
__global__ __launch_bounds__(1024) void k_norm_columns(NormArgs A, int parts) {
  __shared__ float red[64][17];
  const int64_t col = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15);  // of 2 * width, a multiple of 16
  const int k = threadIdx.x >> 4;
  float s = 0.f;
#pragma unroll 8
  for (int i = k; i < parts; i += 64) s += A.part[(int64_t)i * 2 * A.width + col];
  red[k][threadIdx.x & 15] = s;
  __syncthreads();
  // a wave adds the 64 sums of each of its columns
  s = red[threadIdx.x & 63][threadIdx.x >> 6];
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) != 0) return;
  const int64_t to = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 6);
  if (to < A.width) {
    A.dw_pre[to] = s;
    return;
  }
  const int c = (int)(to - A.width);
  if (POST) A.dw_post[c] = GATE == DNB_GATE_VECTOR ? s * ((const float*)A.gate)[c] : s;
  if (GATE == DNB_GATE_VECTOR) ((float*)A.dgate)[c] = POST ? s * A.w_post[c] : s;
}

// Threads a row: a wave up to 1024 values, four up to 8192, sixteen above; NV vectors of 8 a thread.
struct Shape {
  int tpr, nv, rpw;
};
Shape shape_of(int64_t width) {
  const int64_t v = width / 8;
  if (v <= 128) return {64, v <= 64 ? 1 : 2, 4};
  if (v <= 1024) return {256, v <= 256 ? 1 : v <= 512 ? 2 : 4, 1};
  return {1024, 2, 1};
}
int64_t workgroups(int64_t rows, const Shape& s, int64_t most) {
  const int64_t g = (rows + s.rpw - 1) / s.rpw;
  return g < most ? g : most;
}
// The backward pass's workgroups: two on each of 256 compute units, one of 1024 threads; each leaves 2 * width
// partial sums.  (Above width 4096 registers leave room for one of two at a time.)
int64_t backward_workgroups(int64_t rows, const Shape& s) { return workgroups(rows, s, s.tpr == 1024 ? 256 : 512); }

template <typename T, int TPR, int NV, int GATE, bool POST>
hipError_t run(const NormArgs& A, bool back, hipStream_t st) {
  const Shape s = shape_of(A.width);
  const dim3 block(TPR < 256 ? 256 : TPR);
  if (!back) {
    hipLaunchKernelGGL((k_norm_forward<T, TPR, NV, GATE, POST>), dim3((unsigned)workgroups(A.rows, s, 2048)), block, 0, st, A);
    return hipGetLastError();
  }
  const int64_t g = A.rows > 0 ? backward_workgroups(A.rows, s) : 0;
  if (g > 0) {
    hipLaunchKernelGGL((k_norm_backward<T, TPR, NV, GATE, POST>), dim3((unsigned)g), block, 0, st, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_norm_columns<GATE, POST>), dim3((unsigned)(A.width / 8)), dim3(1024), 0, st, A, (int)g * s.rpw);
  return hipGetLastError();
}

template <typename T, int GATE, bool POST>
hipError_t run_width(const NormArgs& A, bool back, hipStream_t st) {
  const Shape s = shape_of(A.width);
  if (s.tpr == 64) return s.nv == 1 ? run<T, 64, 1, GATE, POST>(A, back, st) : run<T, 64, 2, GATE, POST>(A, back, st);
  if (s.tpr == 256)
    return s.nv == 1   ? run<T, 256, 1, GATE, POST>(A, back, st)
           : s.nv == 2 ? run<T, 256, 2, GATE, POST>(A, back, st)
                       : run<T, 256, 4, GATE, POST>(A, back, st);
  return run<T, 1024, 2, GATE, POST>(A, back, st);
}

template <typename T, bool POST>
hipError_t run_gate(const NormArgs& A, int gate, bool back, hipStream_t st) {
  switch (gate) {
    case DNB_GATE_NONE: return run_width<T, DNB_GATE_NONE, POST>(A, back, st);
    case DNB_GATE_VECTOR: return run_width<T, DNB_GATE_VECTOR, POST>(A, back, st);
    default: return run_width<T, DNB_GATE_FULL, POST>(A, back, st);
  }
}

int run_any(const NormArgs& A, int gate, int dtype, bool back, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  hipError_t e;
  if (dtype == DNB_BF16) e = A.w_post ? run_gate<__bf16, true>(A, gate, back, st) : run_gate<__bf16, false>(A, gate, back, st);
  else e = A.w_post ? run_gate<float, true>(A, gate, back, st) : run_gate<float, false>(A, gate, back, st);
  return e == hipSuccess ? DNB_OK : DNB_E_LAUNCH;
}

int check(int64_t rows, int64_t width, float scale, float eps, int gate_kind, int dtype) {
  if (gate_kind != DNB_GATE_NONE && gate_kind != DNB_GATE_VECTOR && gate_kind != DNB_GATE_FULL) return DNB_E_BADDESC;
  if ((dtype != DNB_F32 && dtype != DNB_BF16) || rows < 0 || width < 1 || !(eps >= 0.f) || scale != scale) return DNB_E_BADDESC;
  if (width % 8 != 0) return DNB_E_UNSUPPORTED;
  if (width > 16384 || rows > 0x7fffffff) return DNB_E_RANGE;
  return DNB_OK;
}

}  // namespace

extern "C" {

size_t dnb_op_norm_residual_scratch_bytes(int64_t rows, int64_t width, int gate_kind) {
  if (check(rows, width, 1.f, 0.f, gate_kind, DNB_F32) != DNB_OK) return 0;
  const Shape s = shape_of(width);
  return (size_t)(backward_workgroups(rows, s) * s.rpw * 2 * width) * sizeof(float);
}

int dnb_op_norm_residual_forward(const void* b, const void* r, const float* w_post, const void* gate, const float* w_pre,
                                 void* h_new, void* y, int64_t rows, int64_t width, float scale, float eps, int gate_kind,
                                 int dtype, void* stream) {
  const int rc = check(rows, width, scale, eps, gate_kind, dtype);
  if (rc != DNB_OK) return rc;
  if (rows == 0) return DNB_OK;
  if (!b || !r || !w_pre || !h_new || !y || (gate_kind != DNB_GATE_NONE && !gate)) return DNB_E_NULL;
  for (const void* p : {b, r, (const void*)w_post, gate, (const void*)w_pre, (const void*)h_new, (const void*)y})
    if ((uintptr_t)p & 15) return DNB_E_ALIGN;
  NormArgs A{};
  A.b = b; A.r = r; A.w_post = w_post; A.gate = gate; A.w_pre = w_pre; A.h_new = h_new; A.y = y;
  A.rows = rows; A.width = (int)width; A.scale = scale; A.eps = eps;
  return run_any(A, gate_kind, dtype, false, stream);
}

int dnb_op_norm_residual_backward(const void* b, const void* h_new, const float* w_post, const void* gate, const float* w_pre,
                                  const void* dh, const void* dy, void* db, void* dr, float* dw_post, void* dgate,
                                  float* dw_pre, int64_t rows, int64_t width, float scale, float eps, int gate_kind, int dtype,
                                  void* scratch, void* stream) {
  const int rc = check(rows, width, scale, eps, gate_kind, dtype);
  if (rc != DNB_OK) return rc;
  if (!w_pre || !dw_pre || (w_post && !dw_post) || (gate_kind != DNB_GATE_NONE && (!gate || !dgate) && (rows > 0 || gate_kind == DNB_GATE_VECTOR)))
    return DNB_E_NULL;
  if (rows > 0 && (!b || !h_new || !dh || !dy || !db || !dr || !scratch)) return DNB_E_NULL;
  for (const void* p : {b, h_new, (const void*)w_post, gate, (const void*)w_pre, dh, dy, (const void*)db, (const void*)dr,
                        (const void*)dw_post, (const void*)dgate, (const void*)dw_pre, (const void*)scratch})
    if ((uintptr_t)p & 15) return DNB_E_ALIGN;
  NormArgs A{};
  A.b = b; A.h = h_new; A.w_post = w_post; A.gate = gate; A.w_pre = w_pre; A.dh = dh; A.dy = dy;
  A.db = db; A.dr = dr; A.dw_post = dw_post; A.dgate = dgate; A.dw_pre = dw_pre; A.part = (float*)scratch;
  A.rows = rows; A.width = (int)width; A.scale = scale; A.eps = eps;
  return run_any(A, gate_kind, dtype, true, stream);
}

}  // extern "C"
