// Queries and keys before the attention: each head's norm (root mean square, no mean taken out) and its rotation by the
// row's position in one pass over the rows,
//   n = x / rms(x) * w      a' = factor (a cos - b sin)   b' = factor (b cos + a sin)   for the pairs (a, b) of n
// its gradients,
//   dn = dy turned back     dw = sum over rows and heads of dn x / rms     dx = (dn w - x / rms mean(dn w x / rms)) / rms
// and the form that leaves keys and values in the pages of a cache.
// A head lies in the registers of `lanes` lanes, two vectors of up to 16 bytes each: with DNB_ROPE_HALF vectors u and
// u + half of a head, so that both of a pair are one lane's.  The angles of a workgroup's rows are computed once, into LDS
// (positions times turns in 64 bits).  Queries, keys and values are parts of one launch, each a range of workgroups.
//
// Bound by memory: 16381 rows of 32 + 8 heads of 128 in bf16 61 us forward (336 MB), 122 us backward (503 MB) and 4.5 us for the sums over
// workgroups; 12597 tokens with their values into pages 68 us (310 MB).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <cmath>

#include "dnb_paged.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxAngles = 1024;  // (row, pair) angles of a workgroup in LDS
constexpr int kMaxRows = 64;      // rows of a workgroup at a time
constexpr unsigned kAcross = 1u << 22;
constexpr int kGroups = 1024;     // workgroups of the backward pass, each of which leaves sums (step of 16381 rows 190 us; 1536: 205, 2048: 193)

// One of queries, keys, values.
struct Part {
  const void *x, *dy;
  void *y, *dx;
  const float* w;
  int64_t xs, ys;       // strides of rows of x and dx, y and dy
  int heads, first;     // first: workgroup number of the part's first
  int rows, blocks;     // rows of a workgroup at a time, workgroups
  uint32_t magic;       // j / heads = umulhi(j, magic)
  int turned, paged;
};

struct QkArgs {
  Part part[3];
  const int32_t* pos;
  const double* turns;
  float* sums;          // (workgroup, head_dim)
  float* dw[2];
  int64_t rows;
  int dim, half;        // half: pairs of a head
  int lanes_log;        // lanes of a head, a power of two
  int vecs;             // vectors of a head
  float eps, factor;
  // of a cache
  const int32_t *qo, *lens, *table;
  int64_t pages, page_stride, row_stride, head_stride;
  int sequences, columns, shift;
};

template <typename T, int V>
struct __attribute__((aligned(sizeof(T) * V < 16 ? sizeof(T) * V : 16))) Vec {
  T v[V];
};

// Sum over 2^log lanes side by side, in every one of them.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lanes_sum(float v, int log) {
  if (log > 0) v += dpp<0xb1>(v);   // quad_perm 1 0 3 2
  if (log > 1) v += dpp<0x4e>(v);   // quad_perm 2 3 0 1
  if (log > 2) v += dpp<0x141>(v);  // the other four of eight
  if (log > 3) v += dpp<0x140>(v);  // the other eight of sixteen
  if (log > 4) v += __shfl_xor(v, 16);
  if (log > 5) v += __shfl_xor(v, 32);
  return v;
}

// Where a head's vectors of unit u begin, and whether they are there
template <int V, bool HALF>
struct Unit {
  int e0, e1;
  bool in0, in1, t0, t1;  // there; turned
  __device__ __forceinline__ Unit(const QkArgs& A, int u) {
    const int hv = A.half / V;
    if (HALF && u < hv) {
      e0 = u * V;
      e1 = A.half + u * V;
      in0 = in1 = t0 = t1 = true;
    } else {
      const int rest = HALF ? 2 * hv : 0, n = A.vecs - rest, split = (n + 1) / 2, w = HALF ? u - hv : u;
      in0 = w < split;
      in1 = w + split < n;
      e0 = (rest + w) * V;
      e1 = (rest + w + split) * V;
      t0 = !HALF && in0 && e0 < 2 * A.half;
      t1 = !HALF && in1 && e1 < 2 * A.half;
    }
  }
};

template <typename T, int V>
__device__ __forceinline__ void load(float (&v)[V], const T* p, bool in) {
  if (in) {
    const Vec<T, V> x = *reinterpret_cast<const Vec<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)x.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.f;
  }
}
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const float (&v)[V], bool in) {
  if (!in) return;
  Vec<T, V> x;
#pragma unroll
  for (int i = 0; i < V; ++i) x.v[i] = (T)v[i];
  *reinterpret_cast<Vec<T, V>*>(p) = x;
}

// Turns a unit's two vectors by the row's angles cs; sign -1: back.
template <int V, bool HALF>
__device__ __forceinline__ void turn(const QkArgs& A, const Unit<V, HALF>& U, const float2* cs, float sign, float (&a)[V], float (&b)[V]) {
  if constexpr (HALF) {
    if (!U.t0) return;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float2 t = cs[U.e0 + k];
      const float f = a[k], g = b[k], s = t.y * sign;
      a[k] = f * t.x - g * s;
      b[k] = g * t.x + f * s;
    }
  } else {
    auto side = [&](float (&v)[V], int e) {
#pragma unroll
      for (int k = 0; k + 1 < V; k += 2) {
        const float2 t = cs[(e + k) / 2];
        const float f = v[k], g = v[k + 1], s = t.y * sign;
        v[k] = f * t.x - g * s;
        v[k + 1] = g * t.x + f * s;
      }
    };
    if (U.t0) side(a, U.e0);
    if (U.t1) side(b, U.e1);
  }
}

// The sequence of a row of what is new, by the whole wave; -1: none.  The last whose first row is not past it.
__device__ __forceinline__ int sequence_of(const QkArgs& A, int64_t row) {
  const int l = threadIdx.x & 63;
  int lo = 0, len = A.sequences;
  while (len > 0) {
    const int step = (len + 63) / 64;
    const bool ok = (int64_t)l * step < len && A.qo[lo + l * step] <= row;
    const int n = (int)__popcll(__ballot(ok));
    if (n == 0) return -1;
    lo += (n - 1) * step;
    if (step == 1) break;
    len = min(step, len - (n - 1) * step);
  }
  return A.qo[lo + 1] > row ? lo : -1;
}

// A workgroup's rows: angles, and (with a cache) the places of their tokens.
struct Rows {
  float2 cs[kMaxAngles];
  int64_t to[kMaxRows];  // the token's row in the pool, -1: none, -2: the row is of no sequence
  int32_t pos[kMaxRows];
};

template <bool PAGED>
__device__ __forceinline__ void prepare_rows(const QkArgs& A, const Part& P, Rows& R, int64_t r0, int nr) {
  if constexpr (PAGED) {
    for (int r = threadIdx.x >> 6; r < nr; r += kThreads / 64) {
      const int s = __builtin_amdgcn_readfirstlane(sequence_of(A, r0 + r));
      int64_t to = -2, place = 0;
      if (s >= 0) {
        to = -1;
        const int64_t q0 = max((int64_t)A.qo[s], (int64_t)0), q1 = min((int64_t)A.qo[s + 1], A.rows);
        place = (r0 + r - q0) + (int64_t)A.lens[s] - (q1 - q0);
        if (place >= 0 && (place >> A.shift) < A.columns) {
          const int64_t page = A.table[(int64_t)s * A.columns + (place >> A.shift)];
          if (page >= 0 && page < A.pages) to = page * A.page_stride + (place & ((1 << A.shift) - 1)) * A.row_stride;
        }
      }
      if ((threadIdx.x & 63) == 0) {
        R.to[r] = to;
        R.pos[r] = A.pos ? A.pos[r0 + r] : (int32_t)place;
      }
    }
    __syncthreads();
  }
  if (!P.turned || A.half == 0) return;
  for (int i = threadIdx.x; i < nr * A.half; i += kThreads) {
    const int r = i / A.half, p = i - r * A.half;
    const double t = (double)(PAGED ? R.pos[r] : A.pos[r0 + r]) * A.turns[p];
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    R.cs[i] = make_float2(c * A.factor, s * A.factor);
  }
  __syncthreads();
}

__device__ __forceinline__ const Part& part_of(const QkArgs& A, unsigned id, unsigned* block) {
  const Part& P = (int)id >= A.part[2].first ? A.part[2] : (int)id >= A.part[1].first ? A.part[1] : A.part[0];
  *block = id - P.first;
  return P;
}

// NU: units of a lane
template <typename T, int V, bool HALF, int NU, bool PAGED>
__global__ __launch_bounds__(kThreads) void k_qk_forward(QkArgs A) {
  __shared__ Rows R;
  unsigned block;
  const Part& P = part_of(A, blockIdx.y * kAcross + blockIdx.x, &block);
  const int64_t r0 = (int64_t)block * P.rows;
  if (r0 >= A.rows) return;
  const int nr = (int)min((int64_t)P.rows, A.rows - r0);
  prepare_rows<PAGED>(A, P, R, r0, nr);
  const int lanes = 1 << A.lanes_log, u = threadIdx.x & (lanes - 1), slots = kThreads >> A.lanes_log;
  const int items = nr * P.heads;
  const float inv_d = 1.f / A.dim;
  for (int j = threadIdx.x >> A.lanes_log; j < items; j += slots) {
    const int r = P.heads == 1 ? j : (int)__umulhi((uint32_t)j, P.magic), h = j - r * P.heads;
    const T* x = (const T*)P.x + (r0 + r) * P.xs + (int64_t)h * A.dim;
    T* y = (T*)P.y + (r0 + r) * P.ys + (int64_t)h * A.dim;
    if constexpr (PAGED) {
      const int64_t to = R.to[r];
      if (to == -2 || (P.paged && to < 0)) continue;
      if (P.paged) y = (T*)P.y + to + h * A.head_stride;
    }
    float a[NU][V], b[NU][V], ss = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const Unit<V, HALF> U(A, u + i * lanes);
      load<T, V>(a[i], x + U.e0, U.in0);
      load<T, V>(b[i], x + U.e1, U.in1);
#pragma unroll
      for (int k = 0; k < V; ++k) ss = fmaf(b[i][k], b[i][k], fmaf(a[i][k], a[i][k], ss));
    }
    const bool norm = P.w != nullptr;
    const float inv = norm ? 1.f / sqrtf(lanes_sum(ss, A.lanes_log) * inv_d + A.eps) : 1.f;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const Unit<V, HALF> U(A, u + i * lanes);
      if (norm) {
        float wa[V], wb[V];
        load<float, V>(wa, P.w + U.e0, U.in0);
        load<float, V>(wb, P.w + U.e1, U.in1);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          a[i][k] *= inv * wa[k];
          b[i][k] *= inv * wb[k];
        }
      }
      if (P.turned) turn<V, HALF>(A, U, R.cs + r * A.half, 1.f, a[i], b[i]);
      store<T, V>(y + U.e0, a[i], U.in0);
      store<T, V>(y + U.e1, b[i], U.in1);
    }
  }
}

template <typename T, int V, bool HALF, int NU>
__global__ __launch_bounds__(kThreads) void k_qk_backward(QkArgs A) {
  __shared__ Rows R;
  unsigned block;
  const Part& P = part_of(A, blockIdx.x, &block);
  const int lanes = 1 << A.lanes_log, u = threadIdx.x & (lanes - 1), slots = kThreads >> A.lanes_log;
  const float inv_d = 1.f / A.dim;
  const bool norm = P.w != nullptr;
  float wa[NU][V], wb[NU][V], sa[NU][V], sb[NU][V];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const Unit<V, HALF> U(A, u + i * lanes);
    load<float, V>(wa[i], P.w + U.e0, norm && U.in0);
    load<float, V>(wb[i], P.w + U.e1, norm && U.in1);
#pragma unroll
    for (int k = 0; k < V; ++k) sa[i][k] = sb[i][k] = 0.f;
  }
  for (int64_t r0 = (int64_t)block * P.rows; r0 < A.rows; r0 += (int64_t)P.blocks * P.rows) {
    const int nr = (int)min((int64_t)P.rows, A.rows - r0);
    prepare_rows<false>(A, P, R, r0, nr);
    const int items = nr * P.heads;
    for (int j = threadIdx.x >> A.lanes_log; j < items; j += slots) {
      const int r = P.heads == 1 ? j : (int)__umulhi((uint32_t)j, P.magic), h = j - r * P.heads;
      const int64_t xat = (r0 + r) * P.xs + (int64_t)h * A.dim, yat = (r0 + r) * P.ys + (int64_t)h * A.dim;
      float a[NU][V], b[NU][V], p[NU][V], q[NU][V], ss = 0.f, dot = 0.f;
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const Unit<V, HALF> U(A, u + i * lanes);
        load<T, V>(a[i], (const T*)P.x + xat + U.e0, norm && U.in0);
        load<T, V>(b[i], (const T*)P.x + xat + U.e1, norm && U.in1);
        load<T, V>(p[i], (const T*)P.dy + yat + U.e0, U.in0);
        load<T, V>(q[i], (const T*)P.dy + yat + U.e1, U.in1);
      }
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const Unit<V, HALF> U(A, u + i * lanes);
        turn<V, HALF>(A, U, R.cs + r * A.half, -1.f, p[i], q[i]);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          ss = fmaf(b[i][k], b[i][k], fmaf(a[i][k], a[i][k], ss));
          dot = fmaf(q[i][k] * wb[i][k], b[i][k], fmaf(p[i][k] * wa[i][k], a[i][k], dot));
        }
      }
      float inv = 1.f, m = 0.f;
      if (norm) {
        inv = 1.f / sqrtf(lanes_sum(ss, A.lanes_log) * inv_d + A.eps);
        m = lanes_sum(dot, A.lanes_log) * inv * inv_d;
      }
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const Unit<V, HALF> U(A, u + i * lanes);
        if (norm) {
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const float xa = a[i][k] * inv, xb = b[i][k] * inv;
            sa[i][k] = fmaf(p[i][k], xa, sa[i][k]);
            sb[i][k] = fmaf(q[i][k], xb, sb[i][k]);
            p[i][k] = inv * (p[i][k] * wa[i][k] - xa * m);
            q[i][k] = inv * (q[i][k] * wb[i][k] - xb * m);
          }
        }
        store<T, V>((T*)P.dx + xat + U.e0, p[i], U.in0);
        store<T, V>((T*)P.dx + xat + U.e1, q[i], U.in1);
      }
    }
    __syncthreads();  // the angles have been read
  }
  if (!norm) return;
  // the sums of the workgroup's slots, one value a thread; a slot's sums of all lanes lie side by side
  constexpr int N = 2 * V * NU;
  __shared__ float red[kThreads * N];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const Unit<V, HALF> U(A, u + i * lanes);
    const int at = (threadIdx.x >> A.lanes_log) * A.dim;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (U.in0) red[at + U.e0 + k] = sa[i][k];
      if (U.in1) red[at + U.e1 + k] = sb[i][k];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < A.dim; c += kThreads) {
    float s = 0.f;
    for (int i = 0; i < slots; ++i) s += red[i * A.dim + c];
    A.sums[(int64_t)(P.first + block) * A.dim + c] = s;
  }
}

// Sums over the workgroups of a part, in a fixed order: 16 columns a workgroup, 64 threads a column.
struct Columns {
  const float* sums;
  float *dw[2];
  int first[2], blocks[2], dim;
};
__global__ __launch_bounds__(1024) void k_qk_columns(Columns A) {
  __shared__ float red[64][17];
  const int part = blockIdx.y, col = blockIdx.x * 16 + (threadIdx.x & 15), k = threadIdx.x >> 4;
  if (!A.dw[part]) return;
  float s = 0.f;
  if (col < A.dim) {
#pragma unroll 8
    for (int i = k; i < A.blocks[part]; i += 64) s += A.sums[(int64_t)(A.first[part] + i) * A.dim + col];
  }
  red[k][threadIdx.x & 15] = s;
  __syncthreads();
  s = red[threadIdx.x & 63][threadIdx.x >> 6];
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  const int to = blockIdx.x * 16 + (threadIdx.x >> 6);
  if ((threadIdx.x & 63) == 0 && to < A.dim) A.dw[part][to] = s;
}

// Lanes of a head, rows and workgroups of each part.
void shape(QkArgs& A, int V, int NU, bool backward) {
  A.vecs = A.dim / V;
  const int hv = A.half / V, units = hv + (A.vecs - 2 * hv + 1) / 2;
  A.lanes_log = 0;
  while ((NU << A.lanes_log) < units) ++A.lanes_log;
  const int slots = kThreads >> A.lanes_log;
  int64_t all = 0;
  for (const Part& P : A.part) all += P.heads;
  int first = 0;
  for (Part& P : A.part) {
    P.first = first;
    P.blocks = 0;
    P.rows = 1;
    if (P.heads == 0 || A.rows == 0) continue;
    P.magic = (uint32_t)((0x100000000ull + P.heads - 1) / P.heads);
    // four heads a thread where that leaves enough workgroups, else one: rows' places and angles are found less often (12597 tokens into
    // pages 70 us, 73 with two heads, 75 with one)
    const int64_t want = A.rows * P.heads >= 4ll * slots * 1024 ? 4 * slots : slots;
    int64_t rows = want / P.heads;
    if (A.half > 0 && rows > kMaxAngles / A.half) rows = kMaxAngles / A.half;
    if (rows > kMaxRows) rows = kMaxRows;
    P.rows = rows < 1 ? 1 : (int)rows;
    int64_t blocks = (A.rows + P.rows - 1) / P.rows;
    if (backward) {  // each leaves sums
      const int64_t share = kGroups * P.heads / all;
      blocks = blocks < share ? blocks : share > 0 ? share : 1;
    }
    P.blocks = (int)blocks;
    first += P.blocks;
  }
}

template <typename T, int V, bool HALF, int NU>
hipError_t run(QkArgs A, bool backward, bool paged, hipStream_t st) {
  shape(A, V, NU, backward);
  const int64_t blocks = A.part[2].first + A.part[2].blocks;
  if (!backward) {
    if (blocks == 0) return hipSuccess;
    const dim3 grid((unsigned)(blocks < (int64_t)kAcross ? blocks : kAcross), (unsigned)((blocks + kAcross - 1) / kAcross));
    if (paged) hipLaunchKernelGGL((k_qk_forward<T, V, HALF, NU, true>), grid, dim3(kThreads), 0, st, A);
    else hipLaunchKernelGGL((k_qk_forward<T, V, HALF, NU, false>), grid, dim3(kThreads), 0, st, A);
    return hipGetLastError();
  }
  if (blocks > 0) {
    hipLaunchKernelGGL((k_qk_backward<T, V, HALF, NU>), dim3((unsigned)blocks), dim3(kThreads), 0, st, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!A.dw[0] && !A.dw[1]) return hipSuccess;
  Columns C{A.sums, {A.dw[0], A.dw[1]}, {A.part[0].first, A.part[1].first}, {A.part[0].blocks, A.part[1].blocks}, A.dim};
  hipLaunchKernelGGL(k_qk_columns, dim3((unsigned)((A.dim + 15) / 16), 2), dim3(1024), 0, st, C);
  return hipGetLastError();
}

// Values of a vector: up to 16 bytes, of which rows, heads and the turned part consist wholly
int vector_of(const dnb_qk_layout& d) {
  const int64_t turned = d.order == DNB_ROPE_HALF ? d.rotary_dim / 2 : d.rotary_dim;
  const int64_t all = turned | d.head_dim | d.q_stride | d.k_stride | d.v_stride | d.q_out_stride | d.k_out_stride;
  for (int v = d.dtype == DNB_BF16 ? 8 : 4; v > 1; v /= 2)
    if (all % v == 0) return v;
  return 1;
}

template <typename T>
hipError_t run_type(const QkArgs& A, int V, bool half, bool backward, bool paged, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (V == 8) return half ? run<T, 8, true, 1>(A, backward, paged, st) : run<T, 8, false, 1>(A, backward, paged, st);
  }
  if (V == 4) return half ? run<T, 4, true, 1>(A, backward, paged, st) : run<T, 4, false, 1>(A, backward, paged, st);
  if (V == 2) return half ? run<T, 2, true, 1>(A, backward, paged, st) : run<T, 2, false, 1>(A, backward, paged, st);
  return run<T, 1, true, 2>(A, backward, paged, st);  // (an odd number of pairs, by halves)
}

int check(const dnb_qk_layout* in, dnb_qk_layout* out) {
  if (!in) return DNB_E_NULL;
  dnb_qk_layout d = *in;
  if (d.rows < 0 || d.q_heads < 0 || d.k_heads < 0 || d.q_heads + (int64_t)d.k_heads < 1 || d.head_dim < 1 || d.rotary_dim < 0 ||
      d.rotary_dim % 2 != 0 || d.rotary_dim > d.head_dim || (d.order != DNB_ROPE_HALF && d.order != DNB_ROPE_INTERLEAVED) ||
      (d.dtype != DNB_F32 && d.dtype != DNB_BF16) || !(d.eps >= 0.f && d.eps < INFINITY) || !(fabsf(d.factor) < INFINITY))
    return DNB_E_BADDESC;
  if (d.head_dim % 2 != 0 || d.head_dim > 256) return DNB_E_UNSUPPORTED;
  if (d.rows > (1 << 29) || d.q_heads > 4096 || d.k_heads > 4096) return DNB_E_RANGE;
  const int64_t qd = (int64_t)d.q_heads * d.head_dim, kd = (int64_t)d.k_heads * d.head_dim;
  const int64_t dense[5] = {qd, kd, kd, qd, kd};
  int64_t* strides[5] = {&d.q_stride, &d.k_stride, &d.v_stride, &d.q_out_stride, &d.k_out_stride};
  for (int i = 0; i < 5; ++i) {
    if (*strides[i] == 0) *strides[i] = dense[i];
    if (*strides[i] < dense[i] || *strides[i] % 2 != 0 || *strides[i] > 0x7fffffff) return DNB_E_RANGE;
  }
  *out = d;
  return DNB_OK;
}

QkArgs args_of(const dnb_qk_layout& d, const void* q, const void* k, const float* w_q, const float* w_k, const int32_t* positions,
               const double* turns) {
  QkArgs A{};
  A.rows = d.rows; A.dim = d.head_dim; A.half = d.rotary_dim / 2; A.eps = d.eps; A.factor = d.factor;
  A.pos = positions; A.turns = turns;
  A.part[0].x = q; A.part[0].w = w_q; A.part[0].xs = d.q_stride; A.part[0].ys = d.q_out_stride; A.part[0].heads = d.q_heads;
  A.part[1].x = k; A.part[1].w = w_k; A.part[1].xs = d.k_stride; A.part[1].ys = d.k_out_stride; A.part[1].heads = d.k_heads;
  A.part[0].turned = A.part[1].turned = d.rotary_dim > 0;
  return A;
}

bool odd(const void* p, uintptr_t by) { return ((uintptr_t)p & (by - 1)) != 0; }

int launch(const QkArgs& A, const dnb_qk_layout& d, bool backward, bool paged, void* stream) {
  const int V = vector_of(d);
  const bool half = d.order == DNB_ROPE_HALF;
  const hipError_t e = d.dtype == DNB_BF16 ? run_type<__bf16>(A, V, half, backward, paged, (hipStream_t)stream)
                                           : run_type<float>(A, V, half, backward, paged, (hipStream_t)stream);
  return e == hipSuccess ? DNB_OK : DNB_E_LAUNCH;
}

}  // namespace

extern "C" {

int dnb_op_qk_rope_forward(const dnb_qk_layout* qk, const void* q, const void* k, const float* w_q, const float* w_k,
                           const int32_t* positions, const double* turns, void* q_out, void* k_out, void* stream) {
  dnb_qk_layout d;
  const int rc = check(qk, &d);
  if (rc != DNB_OK) return rc;
  if (d.rows == 0) return DNB_OK;
  if ((d.q_heads > 0 && (!q || !q_out)) || (d.k_heads > 0 && (!k || !k_out)) || (d.rotary_dim > 0 && (!positions || !turns))) return DNB_E_NULL;
  for (const void* p : {q, k, (const void*)w_q, (const void*)w_k, (const void*)q_out, (const void*)k_out})
    if (odd(p, 16)) return DNB_E_ALIGN;
  if (odd(turns, 8) || odd(positions, 4)) return DNB_E_ALIGN;
  QkArgs A = args_of(d, q, k, w_q, w_k, positions, turns);
  A.part[0].y = q_out;
  A.part[1].y = k_out;
  return launch(A, d, false, false, stream);
}

size_t dnb_op_qk_rope_scratch_bytes(const dnb_qk_layout* qk) {
  dnb_qk_layout d;
  if (check(qk, &d) != DNB_OK) return 0;
  return (size_t)(kGroups + 2) * d.head_dim * sizeof(float);
}

int dnb_op_qk_rope_backward(const dnb_qk_layout* qk, const void* q, const void* k, const float* w_q, const float* w_k,
                            const int32_t* positions, const double* turns, const void* dq_out, const void* dk_out, void* dq,
                            void* dk, float* dw_q, float* dw_k, void* scratch, void* stream) {
  dnb_qk_layout d;
  const int rc = check(qk, &d);
  if (rc != DNB_OK) return rc;
  if ((w_q && !dw_q) || (w_k && !dw_k)) return DNB_E_NULL;
  if (d.rows > 0) {
    // (x is read for the norm alone)
    if ((d.q_heads > 0 && ((w_q && !q) || !dq_out || !dq)) || (d.k_heads > 0 && ((w_k && !k) || !dk_out || !dk)) ||
        (d.rotary_dim > 0 && (!positions || !turns)) || ((w_q || w_k) && !scratch))
      return DNB_E_NULL;
  }
  for (const void* p : {q, k, (const void*)w_q, (const void*)w_k, dq_out, dk_out, (const void*)dq, (const void*)dk, (const void*)dw_q,
                        (const void*)dw_k, (const void*)scratch})
    if (odd(p, 16)) return DNB_E_ALIGN;
  if (odd(turns, 8) || odd(positions, 4)) return DNB_E_ALIGN;
  QkArgs A = args_of(d, q, k, w_q, w_k, positions, turns);
  A.part[0].dy = dq_out; A.part[0].dx = dq;
  A.part[1].dy = dk_out; A.part[1].dx = dk;
  A.sums = (float*)scratch;
  A.dw[0] = w_q ? dw_q : nullptr;
  A.dw[1] = w_k ? dw_k : nullptr;
  return launch(A, d, true, false, stream);
}

int dnb_op_paged_append(const dnb_qk_layout* qk, const dnb_paged_layout* cache, const void* q, const void* k, const void* v,
                        const float* w_q, const float* w_k, const int32_t* positions, const double* turns, const int32_t* q_offsets,
                        const int32_t* k_lengths, const int32_t* table, void* q_out, void* k_pages, void* v_pages, void* stream) {
  if (!qk || !cache) return DNB_E_NULL;
  dnb_qk_layout d;
  int rc = check(qk, &d);
  if (rc != DNB_OK) return rc;
  dnb_paged_layout c;
  rc = dnb::paged::check_layout(*cache, &c);
  if (rc != DNB_OK) return rc;
  if (c.kv_heads != d.k_heads || c.head_dim != d.head_dim || c.dtype != d.dtype) return DNB_E_BADDESC;
  if (d.rows == 0) return DNB_OK;
  if (!q_offsets || !k_lengths || !table || !k || !v || (c.pages > 0 && (!k_pages || !v_pages)) || (d.q_heads > 0 && (!q || !q_out)) ||
      (d.rotary_dim > 0 && !turns))
    return DNB_E_NULL;
  for (const void* p : {q, k, v, (const void*)w_q, (const void*)w_k, (const void*)q_out, (const void*)k_pages, (const void*)v_pages})
    if (odd(p, 16)) return DNB_E_ALIGN;
  if (odd(turns, 8) || odd(positions, 4) || odd(q_offsets, 4) || odd(k_lengths, 4) || odd(table, 4)) return DNB_E_ALIGN;
  QkArgs A = args_of(d, q, k, w_q, w_k, positions, turns);
  A.part[0].y = q_out;
  A.part[1].y = k_pages;
  A.part[1].paged = 1;
  A.part[2].x = v; A.part[2].xs = d.v_stride; A.part[2].heads = d.k_heads; A.part[2].y = v_pages;
  A.part[2].paged = 1;
  A.qo = q_offsets; A.lens = k_lengths; A.table = table;
  A.pages = c.pages; A.page_stride = c.page_stride; A.row_stride = c.row_stride; A.head_stride = c.head_stride;
  A.sequences = c.sequences; A.columns = c.max_pages; A.shift = dnb::paged::log2_of(c.page_size);
  return launch(A, d, false, true, stream);
}

}  // extern "C"
