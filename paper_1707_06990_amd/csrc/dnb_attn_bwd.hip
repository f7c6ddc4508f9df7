// Attention over packed sequences, backward.  With p = exp(scale q k^T - lse), recomputed, and
// D = sum_d dout * out of a row:
//   dv = p^T dout      ds = p * (dout v^T - D)      dq = scale ds k      dk = scale ds^T q
// Two kernels, so that every gradient is summed by one wave in a fixed order: no atomics, no gradients
// in fp32 in memory, results that repeat bit for bit.  That costs seven matrix products where five would
// do.  k_attn_dq walks over the keys for 32 packed rows a wave and leaves D for k_attn_dkv, which walks
// over the rows of all heads of a group for 32 keys a wave (the sum over shared heads is part of it).
#include <hip/hip_runtime.h>

#include "dnb_attn.h"

namespace dnb {
namespace attn {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 128;  // packed rows, or keys, of a workgroup, 32 a wave

template <typename T, int DB>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void k_attn_dq(Args A) {
  using L = Tile<T, DB>;
  constexpr int KT = L::ROWS, NB = KT / 32;
  extern __shared__ __attribute__((aligned(16))) char lds[];  // [2][K tile, V tile]
  const int g = blockIdx.x % A.kv, l = lane_id(), wave = threadIdx.x >> 6;
  Seq S;
  int t, count;
  if (!find_tile(A, blockIdx.x / A.kv, [&](const Seq& s) { return (int)(((int64_t)s.nq * A.per + kRows - 1) / kRows); }, &S, &t, &count))
    return;
  if (A.causal) t = count - 1 - t;
  const int M = S.nq * A.per, m0 = t * kRows, shift = S.nk - S.nq;
  const int m = m0 + wave * 32 + (l & 31), row = m / A.per, sub = m - row * A.per;
  const bool valid = m < M;
  const int head = g * A.per + sub;
  const int64_t qrow = (int64_t)S.q0 + row;
  const int sees = A.causal ? min(max(row + shift + 1, 0), S.nk) : S.nk;
  const int w0 = m0 + wave * 32, w1 = min(w0 + 31, M - 1);
  const int most = w0 >= M ? 0 : A.causal ? min(max(w1 / A.per + shift + 1, 0), S.nk) : S.nk;
  const int least = A.causal ? min(max(w0 / A.per + shift + 1, 0), S.nk) : S.nk;
  const int all = A.causal ? min(max(min(m0 + kRows - 1, M - 1) / A.per + shift + 1, 0), S.nk) : S.nk;

  Piece qf[L::NS], df[L::NS];
  load_cols<T, DB>(qf, (const T*)A.q + qrow * A.qs + (int64_t)head * A.d, valid, A.d);
  load_cols<T, DB>(df, (const T*)A.dout + qrow * A.os + (int64_t)head * A.d, valid, A.d);
  // D of this lane's row: each half of the wave has half of the pieces
  float D = 0.f;
  {
    const T* o = (const T*)A.out + qrow * A.os + (int64_t)head * A.d;
#pragma unroll
    for (int k = 0; k < L::NS; ++k) {
      const int e = (2 * k + (l >> 5)) * L::EP;
      Piece x;
      x.q = (u32x4){0u, 0u, 0u, 0u};
      if (valid && e < A.d) x.q = *reinterpret_cast<const u32x4*>(o + e);
#pragma unroll
      for (int j = 0; j < L::EP; ++j) {
        if constexpr (L::BF) D = fmaf((float)x.b[j], (float)df[k].b[j], D);
        else D = fmaf(x.f[j], df[k].f[j], D);
      }
    }
    D = half_sum(D);
  }
  // lse = -inf: the row sees no key, and none of its p may be anything but 0
  float lse2 = INFINITY;
  if (valid) {
    const float v = A.lse[(int64_t)head * A.rq + qrow];
    if (v != -INFINITY) lse2 = v * kLog2e;
    if (l < 32) A.rowdot[(int64_t)head * A.rq + qrow] = D;
  }
  f32x16 acc[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) acc[i] = (f32x16){};
  const T* kb = (const T*)A.k + (int64_t)S.k0 * A.ks + (int64_t)g * A.d;
  const T* vb = (const T*)A.v + (int64_t)S.k0 * A.vs + (int64_t)g * A.d;
  Stage<T, DB, KT, kThreads> sk, sv;
  sk.init(threadIdx.x, A.ks, A.d);
  sv.init(threadIdx.x, A.vs, A.d);
  auto fetch = [&](int k0) {
    sk.load(kb + (int64_t)k0 * A.ks, A.ks, S.nk - k0, A.d);
    sv.load(vb + (int64_t)k0 * A.vs, A.vs, S.nk - k0, A.d);
  };
  auto put = [&](int buf) {
    sk.store(lds + buf * 2 * L::BYTES, threadIdx.x);
    sv.store(lds + buf * 2 * L::BYTES + L::BYTES, threadIdx.x);
  };
  if (all > 0) {
    fetch(0);
    put(0);
  }
  __syncthreads();
  int buf = 0;
  for (int k0 = 0; k0 < all; k0 += KT, buf ^= 1) {
    if (k0 + KT < all) fetch(k0 + KT);
    if (k0 < most) {
      const char* kt = lds + buf * 2 * L::BYTES;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x16 s = row_mul<T, DB>(kt, 32 * b, qf);
        const f32x16 dp = row_mul<T, DB>(kt + L::BYTES, 32 * b, df);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], A.c, -lse2)) * (dp[i] - D);
        if (k0 + 32 * b + 32 > least) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (k0 + 32 * b + row_of(i) >= sees) s[i] = 0.f;
        }
        col_mul<T, DB>(kt, 32 * b, s, acc);
      }
    }
    if (k0 + KT < all) put(buf ^ 1);
    __syncthreads();
  }
  store_cols<T, DB>((T*)A.dq + qrow * A.qs + (int64_t)head * A.d, valid, A.d, acc, A.scale);
}

template <typename T, int DB>
__global__ __launch_bounds__(kThreads, 1) void k_attn_dkv(Args A) {
  using L = Tile<T, DB>;
  constexpr int QT = L::ROWS, NB = QT / 32;
  // [2][Q tile, dout tile, lse and D of the rows]
  extern __shared__ __attribute__((aligned(16))) char lds[];
  constexpr int BUF = 2 * L::BYTES + 2 * QT * 4;
  const int g = blockIdx.x % A.kv, l = lane_id(), wave = threadIdx.x >> 6;
  Seq S;
  int t, count;
  if (!find_tile(A, blockIdx.x / A.kv, [&](const Seq& s) { return (s.span + kRows - 1) / kRows; }, &S, &t, &count)) return;
  const int c0 = t * kRows, w0 = c0 + wave * 32, key = w0 + (l & 31), shift = S.nk - S.nq;
  const bool valid = key < S.nk;
  // query i sees key j if j <= i + shift: rows from `first` on see some key of the workgroup
  const int first = A.causal ? min(max(c0 - shift, 0), S.nq) : 0;
  const int tiles = c0 < S.nk ? (S.nq - first + QT - 1) / QT : 0, steps = tiles * A.per;

  const int64_t krow = (int64_t)S.k0 + key;
  Piece kf[L::NS], vf[L::NS];
  load_cols<T, DB>(kf, (const T*)A.k + krow * A.ks + (int64_t)g * A.d, valid, A.d);
  load_cols<T, DB>(vf, (const T*)A.v + krow * A.vs + (int64_t)g * A.d, valid, A.d);
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) dk[i] = dv[i] = (f32x16){};

  Stage<T, DB, QT, kThreads> sq, sd;
  sq.init(threadIdx.x, A.qs, A.d);
  sd.init(threadIdx.x, A.os, A.d);
  float st = 0.f;  // lse of row tid, or D of row tid - QT
  auto fetch = [&](int step) {
    const int sub = step / tiles, r0 = first + (step - sub * tiles) * QT, head = g * A.per + sub;
    const int64_t q0 = (int64_t)S.q0 + r0;
    sq.load((const T*)A.q + q0 * A.qs + (int64_t)head * A.d, A.qs, S.nq - r0, A.d);
    sd.load((const T*)A.dout + q0 * A.os + (int64_t)head * A.d, A.os, S.nq - r0, A.d);
    if ((int)threadIdx.x < 2 * QT) {
      const int r = threadIdx.x & (QT - 1);
      const bool is_lse = (int)threadIdx.x < QT;
      st = is_lse ? INFINITY : 0.f;
      if (r0 + r < S.nq) {
        const float x = (is_lse ? A.lse : A.rowdot)[(int64_t)head * A.rq + q0 + r];
        if (!is_lse) st = x;
        else if (x != -INFINITY) st = x * kLog2e;
      }
    }
  };
  auto put = [&](int buf) {
    char* b = lds + buf * BUF;
    sq.store(b, threadIdx.x);
    sd.store(b + L::BYTES, threadIdx.x);
    if ((int)threadIdx.x < 2 * QT) reinterpret_cast<float*>(b + 2 * L::BYTES)[threadIdx.x] = st;
  };
  if (steps > 0) {
    fetch(0);
    put(0);
  }
  __syncthreads();
  int buf = 0, tile = 0;
  for (int step = 0; step < steps; ++step, buf ^= 1) {
    if (step + 1 < steps) fetch(step + 1);
    const char* qt = lds + buf * BUF;
    const char* dt = qt + L::BYTES;
    const float* rows = reinterpret_cast<const float*>(dt + L::BYTES);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int r0 = first + tile * QT + 32 * b;
      // uniform in the wave: some row of the block sees some key of the wave
      if (w0 < S.nk && r0 < S.nq && (!A.causal || r0 + 31 + shift >= w0)) {
        f32x16 s = row_mul<T, DB>(qt, 32 * b, kf);
        f32x16 dp = row_mul<T, DB>(dt, 32 * b, vf);
        const bool edge = w0 + 32 > S.nk || (A.causal && r0 + shift < w0 + 31);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float4 le = *reinterpret_cast<const float4*>(rows + 32 * b + 8 * q + 4 * (l >> 5));
          const float4 Dd = *reinterpret_cast<const float4*>(rows + QT + 32 * b + 8 * q + 4 * (l >> 5));
          const float le_[4] = {le.x, le.y, le.z, le.w}, D_[4] = {Dd.x, Dd.y, Dd.z, Dd.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[4 * q + j], A.c, -le_[j]));
            s[4 * q + j] = p;
            dp[4 * q + j] = p * (dp[4 * q + j] - D_[j]);
          }
        }
        if (edge) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!valid || (A.causal && r0 + row_of(i) + shift < key)) s[i] = dp[i] = 0.f;
        }
        col_mul<T, DB>(dt, 32 * b, s, dv);
        col_mul<T, DB>(qt, 32 * b, dp, dk);
      }
    }
    if (++tile == tiles) tile = 0;
    if (step + 1 < steps) put(buf ^ 1);
    __syncthreads();
  }
  // rows of the sequence's span that are not in use get zeros
  const bool own = key < S.span;
  store_cols<T, DB>((T*)A.dk + krow * A.ks + (int64_t)g * A.d, own, A.d, dk, A.scale);
  store_cols<T, DB>((T*)A.dv + krow * A.vs + (int64_t)g * A.d, own, A.d, dv, 1.f);
}

template <typename T, int DB>
hipError_t run(const Args& A, hipStream_t st) {
  using L = Tile<T, DB>;
  if (A.rq > 0) {
    const int64_t tiles = (A.rq * A.per + kRows - 1) / kRows + A.n;
    hipLaunchKernelGGL((k_attn_dq<T, DB>), dim3((unsigned)(tiles * A.kv)), dim3(kThreads), 4 * L::BYTES, st, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (A.rk > 0) {
    const int64_t tiles = (A.rk + kRows - 1) / kRows + A.n;
    hipLaunchKernelGGL((k_attn_dkv<T, DB>), dim3((unsigned)(tiles * A.kv)), dim3(kThreads), 4 * L::BYTES + 4 * L::ROWS * 4, st, A);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t run_db(const Args& A, hipStream_t st) {
  switch ((A.d + 31) / 32) {
    case 1: return run<T, 1>(A, st);
    case 2: return run<T, 2>(A, st);
    case 3: return run<T, 3>(A, st);
    default: return run<T, 4>(A, st);
  }
}

}  // namespace

hipError_t launch_backward(const Args& A, bool bf16, hipStream_t st) { return bf16 ? run_db<__bf16>(A, st) : run_db<float>(A, st); }

}  // namespace attn
}  // namespace dnb
