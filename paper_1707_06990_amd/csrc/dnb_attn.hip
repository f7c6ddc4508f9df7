// Attention over packed sequences, forward: softmax(scale q k^T) v for each sequence and head, with
// grouped key/value heads and a causal mask whose last query sees the last key.
//
// k_attn: a wave keeps 32 rows and walks over the keys in tiles that the workgroup's four waves share.
// With grouped heads the `per` query heads of a key/value head are rows of one matrix ("packed rows":
// packed row m is query m / per, head m % per of the group), so a tile of keys serves all of them.
// One pass over the keys, with the running maximum and sum of the softmax (both fp32, in units of
// log 2).  The sum so far and its weights are only rescaled when the maximum has grown by more than
// 8 (a factor of 256, far from anything that fp32 sums lose), which after the first tiles it hardly does.
// 12597 packed tokens of 32 heads of 128 on 8 key/value heads, causal: 367 us, 873 TFLOP/s; matrix cores
// 41% busy and vector units 39%: a wave is at either, and registers allow two waves a SIMD.
//
// k_attn_token / k_attn_join: where few rows would leave most compute units idle (answering: one query a
// request) the work is split over the keys instead.  With one query a request it is bound by reading them: 165 MB
// of keys and values in 35 to 37 us (4.5 to 4.7 TB/s), and 6 us for the join.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>
#include <type_traits>

#include "dnb_attn_dev.h"
#include "dnb_attn.h"

namespace dnb {
namespace attn {
namespace {

constexpr int kThreads = 256;

// fp32 at head_dim 97 to 128: 32 bytes a lane (eight waves: 76; at 65 to 96 12) do not fit the registers and go to scratch.
// KH 2: eight waves, of which the second four take the second of every two tiles of keys; their sums meet at
// the end.  A workgroup then takes half the time, which is what counts where there are few of them.
template <typename T, int DB, int KH>
__global__ __launch_bounds__(kThreads * KH, 2) void k_attn(Args A) {
  using L = Tile<T, DB>;
  using E = elem_t<T>;
  constexpr int KT = L::ROWS, NB = KT / 32, STEP = KT * KH, NT = kThreads * KH;
  constexpr bool HOLD = L::PL == 1 || DB <= 2;
  constexpr int BUFS = buffers<T>(DB);
  extern __shared__ __attribute__((aligned(512))) char shared[];  // [BUFS][K tiles, V tiles]
  const lds_t lds = lds_start(shared);
  const unsigned id = flat_block();
  const int g = id % A.kv, l = lane_id(), wave = (threadIdx.x >> 6) & 3, kh = KH == 1 ? 0 : (int)(threadIdx.x >> 8);
  Seq S;
  int t, count;
  if (!find_tile(A, id / A.kv, &S, &t, &count)) return;
  if (A.causal) t = count - 1 - t;  // the rows that see most keys go first
  const RowTile R0(A, S, g, t * kRows + wave * 32);
  const unsigned all = RowTile::seen(A, S, min((t + 1) * kRows, S.nq * A.per) - 1);  // keys that the workgroup's last row sees
  const bool valid = R0.valid;
  const int head = R0.head;
  const unsigned sees = R0.sees, most = R0.most, least = R0.least;
  const int64_t qrow = R0.qrow;

  Online<DB> R;
  auto walk = [&](auto form) {
    using F = decltype(form);
    const int tid = apart<F>((int)threadIdx.x);
    Columns<F, DB> qf;
    load_cols<F, DB>(qf, (const E*)A.q + apart<F>(qrow) * A.qs + (int64_t)apart<F>(head) * A.d, valid, A.d);
    R.init();
    const E* kb = (const E*)A.k + (int64_t)S.k0 * A.ks + (int64_t)g * A.d;
    const E* vb = (const E*)A.v + (int64_t)S.k0 * A.vs + (int64_t)g * A.d;
    Stage<F, DB, STEP, NT> sk, sv;
    sk.init(tid, A.ks, A.d);
    sv.init(tid, A.vs, A.d);
    auto fetch = [&](unsigned k0) {
      sk.load(kb + (int64_t)k0 * A.ks, A.ks, S.nk - k0, A.d);
      sv.load(vb + (int64_t)k0 * A.vs, A.vs, S.nk - k0, A.d);
    };
    auto put = [&](int buf) {
      sk.store(lds + buf * 2 * KH * L::BYTES, tid);
      sv.store(lds + (buf * 2 + 1) * KH * L::BYTES, tid);
    };
    if (!is_whole<F> && all > 0) {
      fetch(0);
      put(0);
    }
    __syncthreads();
    auto step = [&](unsigned at, auto which) {
      constexpr int BUF = which;
      const unsigned k0 = at + kh * KT;
      const bool ahead = !is_whole<F> && at + STEP < all;  // Whole holds no tile over its products
      if (is_whole<F>) {
        fetch(at);
        put(BUFS == 1 ? 0 : BUF);
        __syncthreads();
      }
      if (k0 >= most && ahead) fetch(at + STEP);
      if (k0 < most) {
        const lds_t kt = lds + (BUFS == 1 ? 0 : BUF * 2 * KH * L::BYTES) + kh * KT * L::PITCH;
        f32x16 s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = row_mul<F, DB, HOLD, STEP>(kt, 32 * b, qf);
        // four reads of LDS ahead of their products, and the next tile's registers not taken before: 381 -> 367 us
        // for 12597 packed queries of 32 heads
        if constexpr (L::PL == 1) read_ahead<KH == 1 ? 4 : 2, NB * L::NS>();
        if (ahead) fetch(at + STEP);
        if (k0 + KT > least) {
#pragma unroll
          for (int b = 0; b < NB; ++b) hide(s[b], k0 + 32 * b, sees);
        }
        online_step<F, DB, NB, HOLD, STEP>(R, s, A.c, kt + KH * L::BYTES, 0);
      }
      if (ahead) {
        if (BUFS == 1) __syncthreads();
        put(BUFS == 1 ? 0 : BUF ^ 1);
      }
      __syncthreads();
    };
    for (unsigned at = 0; at < all; at += 2 * STEP) {
      step(at, std::integral_constant<int, 0>());
      if (at + STEP < all) step(at + STEP, std::integral_constant<int, 1>());
    }
  };
  walk(T());
  if constexpr (L::PL == 3) {  // (the last step ended with a barrier)
    if (any_wave<4 * KH>(lds + BUFS * 2 * KH * L::BYTES, not_finite(R.o))) walk(Whole());
  }
  if constexpr (KH == 2) {
    // the second half's O in 16-byte pieces, then its m and l; the last step ended with a barrier
    f32x4* to = reinterpret_cast<f32x4*>(shared) + wave * (DB * 4 + 1) * 64 + l;
    if (kh == 1) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) to[(db * 4 + q) * 64] = (f32x4){R.o[db][4 * q], R.o[db][4 * q + 1], R.o[db][4 * q + 2], R.o[db][4 * q + 3]};
      to[DB * 4 * 64] = (f32x4){R.m, R.l, 0.f, 0.f};
    }
    __syncthreads();
    if (kh == 1) return;
    const f32x4 ml = to[DB * 4 * 64];
    const float m = fmaxf(R.m, ml[0]), t = m == -INFINITY ? 0.f : m;
    const float a = __builtin_amdgcn_exp2f(R.m - t), b = __builtin_amdgcn_exp2f(ml[0] - t);
    R.m = m;
    R.l = R.l * a + ml[1] * b;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 x = to[(db * 4 + q) * 64];
#pragma unroll
        for (int k = 0; k < 4; ++k) R.o[db][4 * q + k] = R.o[db][4 * q + k] * a + x[k] * b;
      }
  }
  const float sum = half_sum(R.l);
  store_cols<E, DB>((E*)A.o + qrow * A.os + (int64_t)head * A.d, valid, A.d, R.o, sum == 0.f ? 0.f : 1.f / sum);
  if (valid && l < 32) A.lse[(int64_t)head * A.rq + qrow] = sum == 0.f ? -INFINITY : (R.m + log2f(sum)) * kLn2;
}

// ---------------------------------------------------------------- work split over the keys

template <typename T, int DB>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void k_attn_token(Args A) {
  using L = Tile<T, DB>;
  extern __shared__ __attribute__((aligned(512))) char shared[];  // a K and a V tile of 32 keys for each wave
  const lds_t lds = lds_start(shared);
  const int l = lane_id(), wave = threadIdx.x >> 6;
  const lds_t kt = lds + wave * 2 * kUnit * L::PITCH, vt = kt + kUnit * L::PITCH;
  Stage<T, DB, kUnit, 64> sk, sv;
  sk.init(l, A.ks, A.d);
  sv.init(l, A.vs, A.d);
  each_part(A, (int64_t)blockIdx.x * 4 + wave, [&](const Seq& S, int g, int m0, int first, int last, int64_t slot) {
    const RowTile R0(A, S, g, m0);
    Columns<T, DB> qf;
    load_cols<T, DB>(qf, (const T*)A.q + R0.qrow * A.qs + (int64_t)R0.head * A.d, R0.valid, A.d);
    Online<DB> R;
    R.init();
    const T* kb = (const T*)A.k + (int64_t)S.k0 * A.ks + (int64_t)g * A.d;
    const T* vb = (const T*)A.v + (int64_t)S.k0 * A.vs + (int64_t)g * A.d;
    auto fetch = [&](int u) {
      sk.load(kb + (int64_t)u * kUnit * A.ks, A.ks, S.nk - u * kUnit, A.d);
      sv.load(vb + (int64_t)u * kUnit * A.vs, A.vs, S.nk - u * kUnit, A.d);
    };
    const int end = min(last, units_of(R0.most));  // no row of the tile sees what follows
    if (first < end) fetch(first);
    for (int u = first; u < end; ++u) {
      // the tiles are this wave's own, and LDS serves a wave's accesses in their order
      sk.store(kt, l);
      sv.store(vt, l);
      if (u + 1 < end) fetch(u + 1);
      __builtin_amdgcn_wave_barrier();
      f32x16 s[1] = {row_mul<T, DB, false, kUnit>(kt, 0, qf)};
      if ((u + 1u) * kUnit > R0.least) hide(s[0], u * kUnit, R0.sees);
      online_step<T, DB, 1, false, kUnit>(R, s, A.c, vt, 0);
      __builtin_amdgcn_wave_barrier();
    }
    float* p = A.part + slot * slot_floats(32 * DB);
    store_cols<float, DB>(p + (l & 31) * 32 * DB, R0.valid, 32 * DB, R.o, 1.f);
    const float sum = half_sum(R.l);
    if (R0.valid && l < 32) {
      p[kItemRows * 32 * DB + l] = R.m;
      p[kItemRows * 32 * DB + kItemRows + l] = sum;
    }
  });
}

// Joins an item's parts: a workgroup for each (query row, head).  32 lanes (at head_dim 128) hold a row and
// eight such groups take every eighth part, each with its own running maximum, so that all of its reads are
// on their way at once: a part comes from another XCD, which takes some 2 us, and a wave that went through
// 51 parts of a row 8 at a time took 20 us.
template <typename T, int DB>
__global__ __launch_bounds__(kThreads) void k_attn_join(Args A) {
  constexpr int DP = 32 * DB, LANES = DP / 4, G = kThreads / LANES;
  __shared__ float red[G][DP + 2];
  const RowParts P = row_parts(A, flat_block());
  if (!P.found) return;  // a row of no sequence
  const int grp = threadIdx.x / LANES, c = threadIdx.x - grp * LANES;
  float M = -INFINITY, sum = 0.f;
  f32x4 o = {};
  if (grp < G) {
    const float* p = A.part + P.slot * slot_floats(DP);
#pragma unroll 8
    for (int i = grp; i < P.n; i += G) {
      const float* q = p + i * slot_floats(DP);
      const f32x4 v = *reinterpret_cast<const f32x4*>(q + P.r * DP + 4 * c);
      const float mi = q[kItemRows * DP + P.r], li = q[kItemRows * DP + kItemRows + P.r];
      const float top = fmaxf(M, mi), t = top == -INFINITY ? 0.f : top;
      const float a = __builtin_amdgcn_exp2f(M - t), b = __builtin_amdgcn_exp2f(mi - t);
      M = top;
      sum = sum * a + li * b;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = o[k] * a + v[k] * b;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) red[grp][4 * c + k] = o[k];
    if (c == 0) {
      red[grp][DP] = M;
      red[grp][DP + 1] = sum;
    }
  }
  __syncthreads();
  if (threadIdx.x >= DP) return;
  M = -INFINITY;
#pragma unroll
  for (int i = 0; i < G; ++i) M = fmaxf(M, red[i][DP]);
  const float t = M == -INFINITY ? 0.f : M;
  sum = 0.f;
  float y = 0.f;
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const float f = __builtin_amdgcn_exp2f(red[i][DP] - t);
    sum = fmaf(red[i][DP + 1], f, sum);
    y = fmaf(red[i][threadIdx.x], f, y);
  }
  if ((int)threadIdx.x < A.d) ((T*)A.o)[P.qrow * A.os + (int64_t)P.head * A.d + threadIdx.x] = (T)(sum == 0.f ? 0.f : y / sum);
  if (threadIdx.x == 0) A.lse[(int64_t)P.head * A.rq + P.qrow] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
}

template <typename T, int DB>
hipError_t run_forward(const Args& A, bool token, hipStream_t st) {
  if (A.index) {
    hipLaunchKernelGGL(k_attn_index<RowSums>, dim3(1), dim3(kIndexThreads), 0, st, A, (int64_t*)A.index);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (token) {
    constexpr int PITCH = Tile<T, DB>::PITCH;
    hipLaunchKernelGGL((k_attn_token<T, DB>), dim3(A.waves / 4), dim3(kThreads), 8 * kUnit * PITCH, st, A);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_attn_join<T, DB>), flat_grid(A.rq * A.heads), dim3(kThreads), 0, st, A);
    return hipGetLastError();
  }
  using M = typename std::conditional<std::is_same<T, float>::value, Split, T>::type;
  constexpr int BYTES = Tile<M, DB>::BYTES, FLAGS = in_parts<M> ? kFlags : 0;
  const int64_t tiles = (A.rq * A.per + kRows - 1) / kRows + A.n;
  if (split_keys(A, tiles))
    hipLaunchKernelGGL((k_attn<M, DB, 2>), flat_grid(tiles * A.kv), dim3(2 * kThreads), 4 * buffers<M>(DB) * BYTES + FLAGS, st, A);
  else
    hipLaunchKernelGGL((k_attn<M, DB, 1>), flat_grid(tiles * A.kv), dim3(kThreads), 2 * buffers<M>(DB) * BYTES + FLAGS, st, A);
  return hipGetLastError();
}

template <typename T>
hipError_t run_forward_db(const Args& A, bool token, hipStream_t st) {
  switch ((A.d + 31) / 32) {
    case 1: return run_forward<T, 1>(A, token, st);
    case 2: return run_forward<T, 2>(A, token, st);
    case 3: return run_forward<T, 3>(A, token, st);
    default: return run_forward<T, 4>(A, token, st);
  }
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace attn
}  // namespace dnb

using namespace dnb::attn;

struct dnb_attn {
  dnb_attn_desc d;
  bool token;       // the forward's form
  int waves;        // of the token form
  int64_t slots;
  size_t ws_index, ws_part, ws_rowdot, ws_bytes;
};

namespace {

void fill(const dnb_attn* p, void* workspace, bool backward, Args* A) {
  const dnb_attn_desc& d = p->d;
  *A = Args{};
  A->n = d.sequences; A->heads = d.heads; A->kv = d.kv_heads; A->per = d.heads / d.kv_heads; A->d = d.head_dim;
  A->causal = d.causal != 0;
  A->rq = d.rows_q; A->rk = d.rows_k; A->qs = d.q_stride; A->ks = d.k_stride; A->vs = d.v_stride;
  A->os = (int64_t)d.heads * d.head_dim;
  A->scale = d.scale;
  A->c = d.scale * kLog2e;
  A->waves = p->waves;
  A->slots = p->slots;
  char* ws = (char*)workspace;
  A->rowdot = (float*)(ws + p->ws_rowdot);
  A->index = d.sequences > (p->token ? kScanSplit : backward ? kScanBackward : kScanForward) ? (const int64_t*)(ws + p->ws_index) : nullptr;
  A->part = (float*)(ws + p->ws_part);
}

}  // namespace

extern "C" {

int dnb_attn_create(const dnb_attn_desc* desc, dnb_attn** out) {
  if (!desc || !out) return DNB_E_NULL;
  dnb_attn_desc d = *desc;
  if (d.heads < 1 || d.kv_heads < 1 || d.heads % d.kv_heads != 0 || d.head_dim < 1 || d.sequences < 1 || d.rows_q < 0 ||
      d.rows_k < 0 || (d.dtype != DNB_F32 && d.dtype != DNB_BF16) || !(d.scale >= 0.f && d.scale < INFINITY))
    return DNB_E_BADDESC;
  if (d.head_dim % 8 != 0 || d.head_dim > 128) return DNB_E_UNSUPPORTED;
  if (d.heads > 65536 || d.sequences > (1 << 20)) return DNB_E_RANGE;
  const int64_t qd = (int64_t)d.heads * d.head_dim, kd = (int64_t)d.kv_heads * d.head_dim;
  if (d.q_stride == 0) d.q_stride = qd;
  if (d.k_stride == 0) d.k_stride = kd;
  if (d.v_stride == 0) d.v_stride = kd;
  if (d.scale == 0.f) d.scale = (float)(1.0 / sqrt((double)d.head_dim));
  const int vec = d.dtype == DNB_BF16 ? 8 : 4, per = d.heads / d.kv_heads;
  // rows are read in 16-byte pieces; a tile of up to 128 rows, 127 strides of at most 2^24 bytes, is addressed with 31 bits
  for (const int64_t s : {d.q_stride, d.k_stride, d.v_stride})
    if (s % vec != 0 || s > (1 << 22)) return DNB_E_RANGE;
  if (d.q_stride < qd || d.k_stride < kd || d.v_stride < kd) return DNB_E_RANGE;
  const int64_t most = 0x7fffffff;
  if (d.rows_q > most || d.rows_k > most || d.rows_q * per > most - 256 || d.rows_q * d.heads > most ||
      ((d.rows_q * per + 31) / 32 + d.sequences) * d.kv_heads > most || (d.rows_k / 32 + 1 + d.sequences) * d.kv_heads > most)
    return DNB_E_RANGE;
  dnb_attn* p = new (std::nothrow) dnb_attn();
  if (!p) return DNB_E_NOMEM;
  p->d = d;
  p->token = split_rows(d.rows_q, d.rows_k, d.sequences, d.kv_heads, per, d.dtype == DNB_BF16);
  const int dp = (d.head_dim + 31) / 32 * 32;
  p->waves = d.dtype == DNB_BF16 ? 2048 : 1024;  // 256 compute units, two workgroups of four waves each, fp32 one
  p->slots = p->token ? p->waves + ((d.rows_q * per + kItemRows - 1) / kItemRows + d.sequences) * d.kv_heads : 0;
  p->ws_rowdot = 0;
  p->ws_index = ((size_t)d.rows_q * d.heads * sizeof(float) + 255) / 256 * 256;
  p->ws_part = (p->ws_index + index_bytes(d.sequences) + 255) / 256 * 256;
  const size_t fwd = (size_t)p->slots * slot_floats(dp) * sizeof(float);
  const size_t bwd = backward_part_bytes(d.rows_q, d.rows_k, d.sequences, d.kv_heads, per, d.head_dim, d.dtype == DNB_BF16);
  p->ws_bytes = p->ws_part + (fwd > bwd ? fwd : bwd);
  *out = p;
  return DNB_OK;
}

void dnb_attn_destroy(dnb_attn* p) { delete p; }

size_t dnb_attn_workspace_bytes(const dnb_attn* p) { return p ? p->ws_bytes : 0; }

int dnb_attn_forward(const dnb_attn* p, const void* q, const void* k, const void* v, const int32_t* q_offsets,
                     const int32_t* k_offsets, const int32_t* k_lengths, void* out, float* lse, void* workspace, void* stream) {
  if (!p || !q_offsets || !k_offsets) return DNB_E_NULL;
  if (p->d.rows_q == 0) return DNB_OK;
  if (!q || !out || !lse || !workspace || (p->d.rows_k > 0 && (!k || !v))) return DNB_E_NULL;
  for (const void* x : {q, k, v, (const void*)out, (const void*)workspace})
    if (!aligned16(x)) return DNB_E_ALIGN;
  Args A;
  fill(p, workspace, false, &A);
  A.q = q; A.k = k; A.v = v; A.o = out; A.lse = lse;
  A.qo = q_offsets; A.ko = k_offsets; A.kl = k_lengths;
  hipStream_t st = (hipStream_t)stream;
  const hipError_t e = p->d.dtype == DNB_BF16 ? run_forward_db<__bf16>(A, p->token, st) : run_forward_db<float>(A, p->token, st);
  return e == hipSuccess ? DNB_OK : DNB_E_LAUNCH;
}

int dnb_attn_backward(const dnb_attn* p, const void* q, const void* k, const void* v, const void* out, const float* lse,
                      const void* dout, const int32_t* q_offsets, const int32_t* k_offsets, const int32_t* k_lengths, void* dq,
                      void* dk, void* dv, void* workspace, void* stream) {
  if (!p || !q_offsets || !k_offsets) return DNB_E_NULL;
  const bool anyq = p->d.rows_q > 0, anyk = p->d.rows_k > 0;
  if (anyq && (!q || !out || !lse || !dout || !dq || !workspace)) return DNB_E_NULL;
  if (anyk && (!k || !v || !dk || !dv || (p->d.sequences > kScanSplit && !workspace))) return DNB_E_NULL;
  for (const void* x : {q, k, v, out, dout, (const void*)dq, (const void*)dk, (const void*)dv, (const void*)workspace})
    if (!aligned16(x)) return DNB_E_ALIGN;
  Args A;
  fill(p, workspace, true, &A);
  A.q = q; A.k = k; A.v = v; A.out = out; A.lse = (float*)lse; A.dout = dout;
  A.dq = dq; A.dk = dk; A.dv = dv;
  A.qo = q_offsets; A.ko = k_offsets; A.kl = k_lengths;
  const hipError_t e = launch_backward(A, p->d.dtype == DNB_BF16, p->token, (hipStream_t)stream);
  return e == hipSuccess ? DNB_OK : DNB_E_LAUNCH;
}

}  // extern "C"
