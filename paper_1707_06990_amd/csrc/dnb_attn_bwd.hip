// Attention over packed sequences, backward.  With p = exp(scale q k^T - lse), recomputed, and
// D = sum_d dout * out of a row:
//   dv = p^T dout      ds = p * (dout v^T - D)      dq = scale ds k      dk = scale ds^T q
// Two kernels, so that every gradient is summed in an order that does not change (by one wave; where waves or
// workgroups share the work of a tile, their sums are added one after another): no atomics, results that
// repeat bit for bit, and no fp32 gradients in memory but those shared sums.  That costs seven matrix products
// where five would do.  k_attn_dq walks over the keys for 32 packed rows a wave and leaves D for k_attn_dkv, which
// walks over the rows of all heads of a group for 32 keys a wave (the sum over shared heads is part of it).
// 7185 packed tokens of 16 heads of 128 on 4 key/value heads, causal: 106 us for dq, 164 us for dk and dv and 16
// for their join.  Both are bound by the chain products - exponentials - products of the two waves that fit a SIMD.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "dnb_attn.h"

namespace dnb {
namespace attn {
namespace {

constexpr int kThreads = 256;

// bf16: where a row sees few keys its ds is large, and two roundings show in it.  Rows that see up to this many
// keys therefore
//  - multiply what rounding ds to bf16 left as well, in dq and dk;
//  - take D from sum_j p_j (dout v^T)_j, which it equals, and not from out, whose rounding is then as large as
//    ds: one more pass over their few keys (k_attn_dq, where a whole workgroup's rows are such rows).
// dq and dk of some ten tokens are 1.1 times as far from the exact gradient as its rounding to bf16 alone, of 33
// tokens 1.4 times, where both were 1.6 times without; a step of 7185 packed tokens takes 3% longer.
constexpr int kFineKeys = 128;

// Two rows of registers for q and dout: above head_dim 64 Split takes those of two waves.  Up to 64 it fits two waves a
// SIMD but for 20 bytes a lane (eight waves: 72) that go to scratch.
template <typename T>
constexpr bool crowded(int blocks) { return in_parts<T> && blocks > 2; }

// KH 2: eight waves, of which the second four take the second of every two tiles of keys (see k_attn).
template <typename T, int DB, int KH>
__global__ __launch_bounds__(kThreads * KH, crowded<T>(DB) ? 1 : 2) void k_attn_dq(Args A) {
  using L = Tile<T, DB>;
  using E = elem_t<T>;
  constexpr int KT = L::ROWS, NB = KT / 32, STEP = KT * KH, NT = kThreads * KH;
  constexpr bool HOLD = DB <= (L::PL == 1 && KH == 1 ? 3 : 2);
  extern __shared__ __attribute__((aligned(512))) char shared[];  // [2][K tiles, V tiles]
  const lds_t lds = lds_start(shared);
  const unsigned id = flat_block();
  const int g = id % A.kv, l = lane_id(), wave = (threadIdx.x >> 6) & 3, kh = KH == 1 ? 0 : (int)(threadIdx.x >> 8);
  Seq S;
  int t, count;
  if (!find_tile(A, id / A.kv, &S, &t, &count)) return;
  if (A.causal) t = count - 1 - t;
  const RowTile R0(A, S, g, t * kRows + wave * 32);
  const unsigned all = RowTile::seen(A, S, min((t + 1) * kRows, S.nq * A.per) - 1);  // keys that the workgroup's last row sees
  const bool valid = R0.valid;
  const int head = R0.head;
  const unsigned sees = R0.sees, most = R0.most, least = R0.least;
  const int64_t qrow = R0.qrow;

  f32x16 acc[DB];
  auto walk = [&](auto form) {
    using F = decltype(form);
    const int tid = apart<F>((int)threadIdx.x), h = apart<F>(head);
    const int64_t at = apart<F>(qrow) * A.os + (int64_t)h * A.d;
    Columns<F, DB> qf, df;
    load_cols<F, DB>(qf, (const E*)A.q + apart<F>(qrow) * A.qs + (int64_t)h * A.d, valid, A.d);
    load_cols<F, DB>(df, (const E*)A.dout + at, valid, A.d);
    float D = dot_rows<T, DB>((const E*)A.out + at, (const E*)A.dout + at, valid, A.d);
    // lse = -inf: the row sees no key, and none of its p may be anything but 0
    float lse2 = INFINITY;
    if (valid) {
      const float v = A.lse[(int64_t)h * A.rq + apart<F>(qrow)];
      if (v != -INFINITY) lse2 = v * kLog2e;
    }
    const bool fine = sizeof(E) == 2 && most <= kFineKeys;
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = (f32x16){};
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
    if (sizeof(E) == 2 && all <= kFineKeys) {  // uniform in the workgroup: D from p and dout v^T
      float d = 0.f;
      for (unsigned at = 0; at < all; at += STEP) {
        fetch(at);
        put(0);
        __syncthreads();
        const unsigned k0 = at + kh * KT;
        const lds_t kt = lds + kh * KT * L::PITCH;
#pragma unroll 1
        for (int b = 0; b < NB && k0 < most; ++b) {
          const f32x16 s = row_mul<F, DB, false, STEP>(kt, 32 * b, qf);
          const f32x16 dp = row_mul<F, DB, false, STEP>(kt + KH * L::BYTES, 32 * b, df);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            d += k0 + 32 * b + row_of(i) >= sees ? 0.f : __builtin_amdgcn_exp2f(fmaf(s[i], A.c, -lse2)) * dp[i];
        }
        __syncthreads();
      }
      D = half_sum(d);
      if constexpr (KH == 2) {  // the other half of the waves has the other tiles
        lds_write(lds + 4 * threadIdx.x, D);
        __syncthreads();
        D += lds_read<float>(lds + 4 * (threadIdx.x ^ 256));
        __syncthreads();
      }
    }
    if (valid && l < 32 && kh == 0) A.rowdot[(int64_t)h * A.rq + apart<F>(qrow)] = D;
    if (!is_whole<F> && all > 0) {
      fetch(0);
      put(0);
    }
    __syncthreads();
    auto step = [&](unsigned at, auto which) {
      constexpr int BUF = which;
      const unsigned k0 = at + kh * KT;
      const bool ahead = !is_whole<F> && at + STEP < all;  // (as in k_attn)
      if (is_whole<F>) {
        fetch(at);
        put(BUF);
        __syncthreads();
      }
      if (k0 >= most && ahead) fetch(at + STEP);
      if (k0 < most) {
        const lds_t kt = lds + BUF * 2 * KH * L::BYTES + kh * KT * L::PITCH;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          f32x16 s = row_mul<F, DB, HOLD, STEP>(kt, 32 * b, qf);
          const f32x16 dp = row_mul<F, DB, HOLD, STEP>(kt + KH * L::BYTES, 32 * b, df);
          if constexpr (L::PL == 1) read_ahead<4, 2 * L::NS>();  // (as in k_attn)
          if (b == 0 && ahead) fetch(at + STEP);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], A.c, -lse2)) * (dp[i] - D);
          if (k0 + 32 * b + 32 > least) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = k0 + 32 * b + row_of(i) >= sees ? 0.f : s[i];
          }
          col_mul<F, DB, HOLD, STEP>(kt, 32 * b, s, acc);
          if (fine) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] -= (float)(__bf16)s[i];
            col_mul<F, DB, HOLD, STEP>(kt, 32 * b, s, acc);
          }
        }
      }
      if (ahead) put(BUF ^ 1);
      __syncthreads();
    };
    for (unsigned at = 0; at < all; at += 2 * STEP) {
      step(at, std::integral_constant<int, 0>());
      if (at + STEP < all) step(at + STEP, std::integral_constant<int, 1>());
    }
  };
  walk(T());
  if constexpr (L::PL == 3) {  // (the last step ended with a barrier)
    if (any_wave<4 * KH>(lds + 4 * KH * L::BYTES, not_finite(acc))) walk(Whole());
  }
  if constexpr (KH == 2) {
    f32x4* to = reinterpret_cast<f32x4*>(shared) + wave * DB * 4 * 64 + l;
    if (kh == 1) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) to[(db * 4 + q) * 64] = (f32x4){acc[db][4 * q], acc[db][4 * q + 1], acc[db][4 * q + 2], acc[db][4 * q + 3]};
    }
    __syncthreads();
    if (kh == 1) return;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 x = to[(db * 4 + q) * 64];
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[db][4 * q + k] += x[k];
      }
  }
  store_cols<E, DB>((E*)A.dq + qrow * A.qs + (int64_t)head * A.d, valid, A.d, acc, A.scale);
}

// k_attn_dq with the work split over the keys (see each_part): a wave's own tiles of 32 keys, and sums of parts
// that k_attn_dq_join adds.
template <typename T, int DB>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 && DB <= 2 ? 2 : 1) void k_attn_dq_token(Args A) {
  using L = Tile<T, DB>;
  const int l = lane_id(), wave = threadIdx.x >> 6;
  const lds_t kt = wave * 2 * kUnit * L::PITCH, vt = kt + kUnit * L::PITCH;
  Stage<T, DB, kUnit, 64> sk, sv;
  sk.init(l, A.ks, A.d);
  sv.init(l, A.vs, A.d);
  each_part(A, (int64_t)blockIdx.x * 4 + wave, [&](const Seq& S, int g, int m0, int first, int last, int64_t slot) {
    const RowTile R(A, S, g, m0);
    const int64_t at = R.qrow * A.os + (int64_t)R.head * A.d;
    Columns<T, DB> qf, df;
    load_cols<T, DB>(qf, (const T*)A.q + R.qrow * A.qs + (int64_t)R.head * A.d, R.valid, A.d);
    load_cols<T, DB>(df, (const T*)A.dout + at, R.valid, A.d);
    float D = dot_rows<T, DB>((const T*)A.out + at, (const T*)A.dout + at, R.valid, A.d);
    float lse2 = INFINITY;
    if (R.valid) {
      const float v = A.lse[(int64_t)R.head * A.rq + R.qrow];
      if (v != -INFINITY) lse2 = v * kLog2e;
    }
    const bool fine = L::BF && R.most <= kFineKeys;
    f32x16 acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = (f32x16){};
    const T* kb = (const T*)A.k + (int64_t)S.k0 * A.ks + (int64_t)g * A.d;
    const T* vb = (const T*)A.v + (int64_t)S.k0 * A.vs + (int64_t)g * A.d;
    auto fetch = [&](int u) {
      sk.load(kb + (int64_t)u * kUnit * A.ks, A.ks, S.nk - u * kUnit, A.d);
      sv.load(vb + (int64_t)u * kUnit * A.vs, A.vs, S.nk - u * kUnit, A.d);
    };
    const int units = units_of(R.most), end = min(last, units);
    if (fine && first == 0 && last >= units) {  // all of the keys that the tile sees: D from p and dout v^T
      float d = 0.f;
      for (int u = 0; u < end; ++u) {
        fetch(u);
        sk.store(kt, l);
        sv.store(vt, l);
        __builtin_amdgcn_wave_barrier();
        const f32x16 s = row_mul<T, DB, false, kUnit>(kt, 0, qf);
        const f32x16 dp = row_mul<T, DB, false, kUnit>(vt, 0, df);
#pragma unroll
        for (int i = 0; i < 16; ++i) d += (unsigned)(u * kUnit) + row_of(i) >= R.sees ? 0.f : __builtin_amdgcn_exp2f(fmaf(s[i], A.c, -lse2)) * dp[i];
        __builtin_amdgcn_wave_barrier();
      }
      D = half_sum(d);
    }
    if (R.valid && l < 32 && first == 0) A.rowdot[(int64_t)R.head * A.rq + R.qrow] = D;
    if (first < end) fetch(first);
    for (int u = first; u < end; ++u) {
      sk.store(kt, l);
      sv.store(vt, l);
      if (u + 1 < end) fetch(u + 1);
      __builtin_amdgcn_wave_barrier();
      f32x16 s = row_mul<T, DB, false, kUnit>(kt, 0, qf);
      const f32x16 dp = row_mul<T, DB, false, kUnit>(vt, 0, df);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], A.c, -lse2)) * (dp[i] - D);
      if ((u + 1u) * kUnit > R.least) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (unsigned)(u * kUnit) + row_of(i) >= R.sees ? 0.f : s[i];
      }
      col_mul<T, DB, false, kUnit>(kt, 0, s, acc);
      if (fine) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] -= (float)(__bf16)s[i];
        col_mul<T, DB, false, kUnit>(kt, 0, s, acc);
      }
      __builtin_amdgcn_wave_barrier();
    }
    store_cols<float, DB>(A.part + slot * slot_floats(32 * DB) + (l & 31) * 32 * DB, R.valid, 32 * DB, acc, A.scale);
  });
}

// As k_attn_join: groups of lanes with a row's parts in turn, then their sums in LDS.
template <typename T, int DB>
__global__ __launch_bounds__(kThreads) void k_attn_dq_join(Args A) {
  constexpr int DP = 32 * DB, LANES = DP / 4, G = kThreads / LANES;
  __shared__ float red[G][DP];
  const RowParts P = row_parts(A, flat_block());
  if (!P.found) return;
  const int grp = threadIdx.x / LANES, c = threadIdx.x - grp * LANES;
  if (grp < G) {
    f32x4 sum = {};
    const float* p = A.part + P.slot * slot_floats(DP) + P.r * DP + 4 * c;
#pragma unroll 8
    for (int i = grp; i < P.n; i += G) sum += *reinterpret_cast<const f32x4*>(p + i * slot_floats(DP));
#pragma unroll
    for (int k = 0; k < 4; ++k) red[grp][4 * c + k] = sum[k];
  }
  __syncthreads();
  if ((int)threadIdx.x >= A.d) return;
  float y = 0.f;
#pragma unroll
  for (int i = 0; i < G; ++i) y += red[i][threadIdx.x];
  ((T*)A.dq)[P.qrow * A.qs + (int64_t)P.head * A.d + threadIdx.x] = (T)y;
}

// row_mul with the columns in LDS too: rows brow0 .. brow0 + 31 of tile bt, of BR rows
template <typename T, int DB, int TR, int BR>
__device__ __forceinline__ f32x16 row_mul_lds(lds_t tile, int row0, lds_t bt, int brow0) {
  using L = Tile<T, DB>;
  const lds_t at = row_address<T, DB>(row0), bat = row_address<T, DB>(brow0);
  f32x16 s = {};
#pragma unroll
  for (int k = 0; k < L::NS; ++k) {
    Pieces<T, DB> a, b;
#pragma unroll
    for (int p = 0; p < L::PL; ++p) {
      a[p].q = lds_read<u32x4>((at ^ (k << 5)) + (tile + p * TR * L::PITCH));
      b[p].q = lds_read<u32x4>((bat ^ (k << 5)) + (bt + p * BR * L::PITCH));
    }
    mma(s, a, b, (T*)nullptr);
  }
  return s;
}

constexpr int kQRows = 64;      // packed rows of a step of k_attn_dkv

// Keys of an item of k_attn_dkv, 32 for each of two waves.  bf16 above head_dim 96: eight waves and 128
// keys, since the two waves that fit each SIMD have no registers left for more of the rows on their way
// to LDS than a thread of a large workgroup has.  fp32 up to 64: eight, since LDS holds one workgroup's
// tiles; above: four, with k and v in registers, since LDS holds no more than the rows' tiles.  At 97 to 128 they do not
// all fit: 132 bytes a lane go to scratch; 201 us of the 540 that a step over 2264 packed rows of 16/8 heads takes.
constexpr int keys_of(bool bf16, int blocks) { return bf16 ? (blocks == 4 ? 128 : 64) : blocks <= 2 ? 128 : 64; }

// What an item costs beside its rows, in rows: some 5 us, three steps in bf16, one and a half in fp32, whose steps
// are six products for one.  (fp32, 48 / 96 / 160: a step over 2264 packed rows of 16/8 heads of 128, causal, 590 / 540 /
// 530 us, of 64 290 / 283 / 286; 1320 of 4 heads of 64, full, 127 / 128 / 131.)
constexpr int item_cost(bool bf16) { return bf16 ? 192 : 96; }
// Cost of the smallest part worth a workgroup.
constexpr int least_cost(bool bf16) { return item_cost(bf16) + kQRows; }

// Items are (sequence, key/value head, KEYS keys), in that order.  An item's cost is the packed rows that see
// its keys; with a causal mask the first items of a long sequence cost far more than the last, and few
// key/value heads make few items.  So all items lie on one line, as long as they cost, which is cut into
// equal parts, one a workgroup; what several workgroups did of one item k_attn_dkv_join adds.
template <int KEYS, bool BF>
struct KeyLine {
  static constexpr int kItemCost = item_cost(BF);
  int64_t nq, nk, per, tiles, used, full;  // tiles of the span; of those in use; of the latter, those that every row sees
  bool causal;
  __device__ __forceinline__ KeyLine(const Args& A, const Seq& s) {
    nq = s.nq; nk = s.nk; per = A.per; causal = A.causal;
    tiles = ((int64_t)s.span + KEYS - 1) / KEYS;
    used = (nk + KEYS - 1) / KEYS;
    const int64_t shift = nk - nq;
    full = !causal ? used : shift < 0 ? 0 : min(used, shift / KEYS + 1);
  }
  // rows that see some key of tile t
  __device__ __forceinline__ int64_t rows(int64_t t) const { return t >= used ? 0 : (t < full ? nq : min(nq, nk - KEYS * t)) * per; }
  // cost of the tiles before t
  __device__ __forceinline__ int64_t before(int64_t t) const {
    const int64_t u = min(t, used), a = min(u, full);
    return (a * nq + (u - a) * nk - KEYS * ((u - 1) * u - (a - 1) * a) / 2) * per + kItemCost * t;
  }
  // where a cut at x of an item's cost lies in its rows
  __device__ __forceinline__ int64_t cut(int64_t t, int64_t x) const {
    const int64_t r = rows(t);
    if (x >= r + kItemCost) return r;
    return x <= kItemCost ? 0 : (x - kItemCost) / kQRows * kQRows;
  }
};

// Workgroups that take part: none for less than least_cost.
__device__ __forceinline__ int64_t key_parts(int64_t total, int most, bool bf16) {
  return max((int64_t)1, min((int64_t)most, total / least_cost(bf16)));
}
template <int KEYS, bool BF>
struct KeySums {
  static constexpr int N = kSums;
  static __device__ __forceinline__ void sums(const Args& A, const Seq& s, int64_t* v) {
    RowSums::sums(A, s, v);
    const KeyLine<KEYS, BF> k(A, s);
    v[kCost] = k.before(k.tiles) * A.kv;
    v[kKeyItems] = k.tiles * A.kv;
  }
};
template <int KEYS, bool BF>
__device__ __forceinline__ int64_t key_total(const Args& A) {
  if (A.index) return index_of(A, kCost)[chunks_of(A.n)];
  int64_t u = 0;
  for (int i = lane_id(); i < A.n; i += 64) {
    const KeyLine<KEYS, BF> k(A, seq_at(A, i));
    u += k.before(k.tiles) * A.kv;
  }
  return bcast64(wave_scan(u), 63);
}

// The item at position x of the line (x < key_total), and how far into its cost x is; or item number x,
// items -1 if there are fewer.
struct KeyAt {
  Seq s;
  int g;
  int64_t t, lo, item;
};
template <int KEYS, bool BF>
__device__ __forceinline__ KeyAt key_at(const Args& A, int64_t x, bool by_item) {
  const int l = lane_id();
  KeyAt r = {};
  int64_t u0 = 0, i0 = 0;  // cost and items before the 64 sequences at hand
  int base = 0;
  if (A.index) {
    const int c = index_find(index_of(A, by_item ? kKeyItems : kCost), chunks_of(A.n), x);
    base = c * 64;
    u0 = index_of(A, kCost)[c];
    i0 = index_of(A, kKeyItems)[c];
  }
  for (; base < A.n; base += 64) {
    Seq mine = {};
    int64_t cost = 0, items = 0;
    if (base + l < A.n) {
      mine = seq_at(A, base + l);
      const KeyLine<KEYS, BF> k(A, mine);
      cost = k.before(k.tiles) * A.kv;
      items = k.tiles * A.kv;
    }
    const int64_t ue = wave_scan(cost), ie = wave_scan(items);
    const uint64_t past = __ballot((by_item ? i0 + ie : u0 + ue) > x);
    if (past) {
      const int at = __builtin_ctzll(past);
      r.s = bcast(mine, at);
      const KeyLine<KEYS, BF> line(A, r.s);
      if (by_item) {
        const int64_t in = x - i0 - bcast64(ie - items, at);
        r.g = (int)(in / line.tiles);
        r.t = in - r.g * line.tiles;
        r.item = x;
        return r;
      }
      const int64_t head_cost = line.before(line.tiles), in = x - u0 - bcast64(ue - cost, at);
      r.g = (int)(in / head_cost);
      const int64_t off = in - r.g * head_cost;
      // the last tile that starts at or before off, 64 candidates at a time
      for (int64_t span = line.tiles; span > 1;) {
        const int64_t step = (span + 63) / 64;
        r.t += (__popcll(__ballot(l * step < span && line.before(r.t + l * step) <= off)) - 1) * step;
        span = min(step, line.tiles - r.t);
      }
      r.lo = off - line.before(r.t);
      r.item = i0 + bcast64(ie - items, at) + r.g * line.tiles + r.t;
      return r;
    }
    u0 += bcast64(ue, 63);
    i0 += bcast64(ie, 63);
  }
  r.item = -1;
  return r;
}

// Half of the waves takes the first 32 rows of every step, the other half the second, each wave 32 keys;
// the two sums over the rows are added at the end.  k and v stay in LDS, not in registers: with dk and dv (128 registers at head_dim 128)
// that leaves room for two waves on each SIMD, one's exponentials under the other's products.
template <typename T, int DB>
__global__ __launch_bounds__(4 * keys_of(sizeof(elem_t<T>) == 2, DB), crowded<T>(DB) ? 1 : 2) void k_attn_dkv(Args A) {
  using L = Tile<T, DB>;
  using E = elem_t<T>;
  constexpr bool BF = sizeof(E) == 2, COLS = crowded<T>(DB);
  constexpr int KEYS = keys_of(BF, DB), KB = KEYS / 32, NT = 4 * KEYS;
  constexpr int KBYTES = COLS ? 0 : KEYS * L::PITCH * L::PL, QBYTES = kQRows * L::PITCH * L::PL;
  extern __shared__ __attribute__((aligned(512))) char shared[];  // k and v tiles unless COLS, q and dout tiles; lse and D of the rows
  const lds_t kt = lds_start(shared), vt = kt + KBYTES, qt = vt + KBYTES, dt = qt + QBYTES, rows = dt + QBYTES;
  const int l = lane_id(), wave = threadIdx.x >> 6, kb = 32 * (wave & (KB - 1)), per = A.per;
  const bool second = wave >= KB;
  const int qb = second ? 32 : 0;
  // x / per for 0 <= x < 64 + per: a quotient of at most 65 and, at per > 64, less than 2, half a step of
  // 1 / per away from the next whole number, against an fp32 error of 2^-23 of it (per <= 65536)
  const float inv = 1.f / per;
  auto over = [&](int x) { return (int)(((float)x + 0.5f) * inv); };

  const bool whole = A.waves == 0;  // a workgroup an item, not a part of the line
  int64_t w = flat_block(), a = 0, b = 1;
  if (!whole) {
    const int64_t total = key_total<KEYS, BF>(A), W = key_parts(total, A.waves, BF);
    if (w >= W) return;
    // neighbours on the line read the same rows: they go to one of the 8 XCDs, whose workgroups are every 8th
    if (W % 8 == 0) w = (w % 8) * (W / 8) + w / 8;
    a = w * total / W;
    b = (w + 1) * total / W;
  }
  // what the search needs is looked up again for every item: it would not fit the registers beside dk and dv
  while (a < b) {
    {
      const KeyAt at = key_at<KEYS, BF>(A, whole ? w : a, whole);
      if (at.item < 0) return;
      const Seq S = at.s;
      const KeyLine<KEYS, BF> line(A, S);
      const int g = at.g;
      const int64_t t = at.t, lo = at.lo, full = line.before(t + 1) - line.before(t), hi = whole ? full : min(full, lo + b - a), item = at.item;
      a += hi - lo;
      const int64_t slot = lo == 0 && hi == full ? -1 : w + item;  // of a part's sums; -1: the item is whole

      const unsigned c0 = (unsigned)t * KEYS, w0 = c0 + kb, key = w0 + (l & 31), nk = S.nk;
      const int64_t shift = (int64_t)S.nk - S.nq;
      const bool valid = key < nk;
      // query i sees key j if j <= i + shift: rows from `first` on see some key of the item
      const int first = A.causal ? (int)min(max((int64_t)c0 - shift, (int64_t)0), (int64_t)S.nq) : 0;
      // the last query that sees no more than kFineKeys keys
      const int fine_to = A.causal ? (int)min(max(kFineKeys - 1 - shift, (int64_t)-1), (int64_t)INT32_MAX) : S.nk <= kFineKeys ? INT32_MAX : -1;
      const int left = (int)line.cut(t, hi);  // packed rows m0 .. left - 1, counted from query `first` on
      f32x16 dk[DB], dv[DB];
      auto walk = [&](auto form) {
        using F = decltype(form);
        const int tid = apart<F>((int)threadIdx.x);
        int m0 = (int)line.cut(t, lo);
#pragma unroll
        for (int i = 0; i < DB; ++i) dk[i] = dv[i] = (f32x16){};
        __syncthreads();  // the item, or the walk, before is done with LDS
        Columns<F, DB> kf, vf;
        if (COLS) {
          const int64_t krow = (int64_t)S.k0 + key;
          load_cols<F, DB>(kf, (const E*)A.k + krow * A.ks + (int64_t)g * A.d, valid && m0 < left, A.d);
          load_cols<F, DB>(vf, (const E*)A.v + krow * A.vs + (int64_t)g * A.d, valid && m0 < left, A.d);
        } else if (m0 < left) {  // uniform in the workgroup
          Stage<F, DB, KEYS, NT> sk;
          sk.init(tid, A.ks, A.d);
          sk.load((const E*)A.k + ((int64_t)S.k0 + c0) * A.ks + (int64_t)g * A.d, A.ks, S.nk - c0, A.d);
          sk.store(kt, tid);
          sk.init(tid, A.vs, A.d);
          sk.load((const E*)A.v + ((int64_t)S.k0 + c0) * A.vs + (int64_t)g * A.d, A.vs, S.nk - c0, A.d);
          sk.store(vt, tid);
        }
        // the first packed row that sees this lane's key; the wave's first key, its last
        auto first_for = [&](unsigned k) { return A.causal ? (int)min(max(((int64_t)k - shift - first) * per, (int64_t)0), (int64_t)left) : 0; };
        const int need = valid ? first_for(key) : left, need0 = w0 < nk ? first_for(w0) : INT32_MAX, need1 = w0 + 32 > nk ? left : first_for(w0 + 31);
        // the step at hand starts at packed row m0: query q0 of the sequence, head s0 of the group
        int q0 = first + m0 / per, s0 = m0 % per;
        constexpr int U = (kQRows * L::CH + NT - 1) / NT;
        u32x4 rq[U * L::LD], rd[U * L::LD];
        float st = 0.f;  // threads 0 .. 63: lse of a row, 64 .. 127: D
        auto fetch = [&](int m, int q, int s) {
          const auto qr = __builtin_amdgcn_make_buffer_rsrc((E*)A.q + ((int64_t)S.q0 + q) * A.qs + (int64_t)g * per * A.d, 0, 0x7fffffff, 0x00027000);
          const auto dr = __builtin_amdgcn_make_buffer_rsrc((E*)A.dout + ((int64_t)S.q0 + q) * A.os + (int64_t)g * per * A.d, 0, 0x7fffffff, 0x00027000);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int i = tid + u * NT, row = i / L::CH, c = i - row * L::CH;
            const int x = over(s + row), e = (s + row - x * per) * A.d + c * L::EP;
            const bool ok = row < kQRows && m + row < left && c * L::EP < A.d;
            const uint32_t oq = ok ? (uint32_t)(x * (int)A.qs + e) * (uint32_t)sizeof(E) : 0x80000000u;
            const uint32_t od = ok ? (uint32_t)(x * (int)A.os + e) * (uint32_t)sizeof(E) : 0x80000000u;
#pragma unroll
            for (int p = 0; p < L::LD; ++p) {
              rq[u * L::LD + p] = __builtin_amdgcn_raw_buffer_load_b128(qr, oq + 16 * p, 0, 0);
              rd[u * L::LD + p] = __builtin_amdgcn_raw_buffer_load_b128(dr, od + 16 * p, 0, 0);
            }
          }
          if (tid < 2 * kQRows) {
            const int r = tid & (kQRows - 1), x = over(s + r);
            const bool is_lse = tid < kQRows;
            st = is_lse ? INFINITY : 0.f;
            if (m + r < left) {
              const float v = (is_lse ? A.lse : A.rowdot)[(int64_t)(g * per + s + r - x * per) * A.rq + S.q0 + q + x];
              if (!is_lse) st = v;
              else if (v != -INFINITY) st = v * kLog2e;
            }
          }
        };
        if (!is_whole<F> && m0 < left) fetch(m0, q0, s0);
        for (; m0 < left; m0 += kQRows) {
          if (is_whole<F>) fetch(m0, q0, s0);
          __syncthreads();  // the step before is done with the tiles
          store_pieces<F, DB, U, NT, kQRows>(qt, tid, rq);
          store_pieces<F, DB, U, NT, kQRows>(dt, tid, rd);
          if (tid < 2 * kQRows) lds_write(rows + 4 * tid, st);
          __syncthreads();
          // of this wave's rows of the step, the last
          const bool fine = BF && q0 + over(s0 + qb + 31) <= fine_to;
          s0 += kQRows % per;
          q0 += kQRows / per;
          if (s0 >= per) {
            s0 -= per;
            ++q0;
          }
          if (!is_whole<F> && m0 + kQRows < left) fetch(m0 + kQRows, q0, s0);
          // uniform in the wave: some row of the block sees some key of the wave
          if (m0 + qb < left && m0 + qb + 31 >= need0) {
            f32x16 s, dp;
            if constexpr (COLS) {
              s = row_mul<F, DB, false, kQRows>(qt, qb, kf);
              dp = row_mul<F, DB, false, kQRows>(dt, qb, vf);
            } else {
              s = row_mul_lds<F, DB, kQRows, KEYS>(qt, qb, kt, kb);
              dp = row_mul_lds<F, DB, kQRows, KEYS>(dt, qb, vt, kb);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4 le = lds_read<f32x4>(rows + 4 * (qb + 8 * q + 4 * (l >> 5)));
              const f32x4 Dd = lds_read<f32x4>(rows + 4 * (kQRows + qb + 8 * q + 4 * (l >> 5)));
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[4 * q + j], A.c, -le[j]));
                s[4 * q + j] = p;
                dp[4 * q + j] = p * (dp[4 * q + j] - Dd[j]);
              }
            }
            if (m0 + qb < need1) {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const bool sees = m0 + qb + row_of(i) >= need;
                s[i] = sees ? s[i] : 0.f;
                dp[i] = sees ? dp[i] : 0.f;
              }
            }
            col_mul<F, DB, false, kQRows>(dt, qb, s, dv);
            col_mul<F, DB, false, kQRows>(qt, qb, dp, dk);
            if (fine) {
#pragma unroll
              for (int i = 0; i < 16; ++i) dp[i] -= (float)(__bf16)dp[i];
              col_mul<F, DB, false, kQRows>(qt, qb, dp, dk);
            }
          }
        }
      };
      walk(T());
      if constexpr (L::PL == 3) {
        const bool odd_k = not_finite(dk), odd_v = not_finite(dv);
        if (any_wave<2 * KB>(rows + 2 * kQRows * 4, odd_k || odd_v)) walk(Whole());
      }
      // The first half of the waves finishes dk, the second dv: each gives the other sum to its partner.
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        f32x16 keep, give;
        if (second) { keep = dv[db]; give = dk[db]; }
        else { keep = dk[db]; give = dv[db]; }
        dk[db] = keep;
        dv[db] = give;
      }
      constexpr int R = DB > 2 ? DB - 2 : DB;  // blocks at a time: what LDS has room for
#pragma unroll
      for (int d0 = 0; d0 < DB; d0 += R) {
        __syncthreads();
        float4* gives = reinterpret_cast<float4*>(shared) + wave * R * 4 * 64;
        const float4* takes = reinterpret_cast<const float4*>(shared) + (second ? wave - KB : wave + KB) * R * 4 * 64;
#pragma unroll
        for (int db = d0; db < d0 + R && db < DB; ++db)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            gives[((db - d0) * 4 + q) * 64 + l] = make_float4(dv[db][4 * q], dv[db][4 * q + 1], dv[db][4 * q + 2], dv[db][4 * q + 3]);
        __syncthreads();
#pragma unroll
        for (int db = d0; db < d0 + R && db < DB; ++db)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 x = takes[((db - d0) * 4 + q) * 64 + l];
            dk[db][4 * q] += x.x;
            dk[db][4 * q + 1] += x.y;
            dk[db][4 * q + 2] += x.z;
            dk[db][4 * q + 3] += x.w;
          }
      }
      if (slot < 0) {  // rows of the sequence's span that are not in use get zeros
        const int64_t krow = (int64_t)S.k0 + key, to = krow * (second ? A.vs : A.ks) + (int64_t)g * A.d;
        store_cols<E, DB>((E*)(second ? A.dv : A.dk) + to, key < (unsigned)S.span, A.d, dk, second ? 1.f : A.scale);
      } else if (slot < A.slots) {
        float4* part = reinterpret_cast<float4*>(A.part) + (slot * 2 * KB + wave) * DB * 4 * 64;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            part[(db * 4 + q) * 64 + l] = make_float4(dk[db][4 * q], dk[db][4 * q + 1], dk[db][4 * q + 2], dk[db][4 * q + 3]);
      }
    }
  }
}

// Adds the parts of an item that several workgroups share, in the line's order; a workgroup for an item and 32
// of head_dim, so that a long chain of parts (each some 2 us away) is read four at a time.
template <typename T, int DB>
__global__ __launch_bounds__(4 * keys_of(sizeof(T) == 2, DB)) void k_attn_dkv_join(Args A) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int KEYS = keys_of(BF, DB), KB = KEYS / 32;
  const int l = lane_id(), wave = threadIdx.x >> 6;
  const int64_t item = flat_block();
  int64_t u0 = 0, i0 = 0, su = 0, si = 0;
  Seq S = {};
  bool found = false;
  int base = 0, end = A.n;
  if (A.index) {
    const int c = index_find(index_of(A, kKeyItems), chunks_of(A.n), item);
    base = c * 64;
    end = min(base + 64, A.n);
    u0 = index_of(A, kCost)[c];
    i0 = index_of(A, kKeyItems)[c];
  }
  for (; base < end; base += 64) {
    Seq mine = {};
    int64_t cost = 0, items = 0;
    if (base + l < A.n) {
      mine = seq_at(A, base + l);
      const KeyLine<KEYS, BF> k(A, mine);
      cost = k.before(k.tiles) * A.kv;
      items = k.tiles * A.kv;
    }
    const int64_t ue = wave_scan(cost), ie = wave_scan(items);
    const uint64_t past = __ballot(i0 + ie > item);
    if (past && !found) {
      const int at = __builtin_ctzll(past);
      S = bcast(mine, at);
      su = u0 + bcast64(ue - cost, at);
      si = i0 + bcast64(ie - items, at);
      found = true;
    }
    u0 += bcast64(ue, 63);
    i0 += bcast64(ie, 63);
  }
  if (!found) return;
  const KeyLine<KEYS, BF> line(A, S);
  const int64_t total = A.index ? key_total<KEYS, BF>(A) : u0, W = key_parts(total, A.waves, BF);
  const int g = (int)((item - si) / line.tiles);
  const int64_t t = (item - si) - g * line.tiles;
  const int64_t from = su + g * line.before(line.tiles) + line.before(t), to = from + line.before(t + 1) - line.before(t);
  // unit u of the line is workgroup ((u + 1) W - 1) / total's
  const int64_t w0 = ((from + 1) * W - 1) / total, w1 = (to * W - 1) / total;
  if (w0 == w1 || w1 + item >= A.slots) return;
  const int db = blockIdx.z;
  f32x16 sum[1] = {};
#pragma unroll 4
  for (int64_t w = w0; w <= w1; ++w) {
    const f32x4* part = reinterpret_cast<const f32x4*>(A.part) + (((w + item) * 2 * KB + wave) * DB + db) * 4 * 64;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 x = part[q * 64 + l];
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[0][4 * q + k] += x[k];
    }
  }
  const bool second = wave >= KB;
  const unsigned key = (unsigned)t * KEYS + 32 * (wave & (KB - 1)) + (l & 31);
  const int64_t krow = (int64_t)S.k0 + key, at = krow * (second ? A.vs : A.ks) + (int64_t)g * A.d + 32 * db;
  store_cols<T, 1>((T*)(second ? A.dv : A.dk) + at, key < (unsigned)S.span, A.d - 32 * db, sum, second ? 1.f : A.scale);
}

// How k_attn_dkv is launched.  Up to 512 packed rows (8 steps an item) a workgroup takes an item: a launch
// less, 13 us for a sequence of 33 rows where the line and its join took 16.  Otherwise the line, in as many
// parts as 256 compute units hold workgroups at once: one each of eight waves, or of four that take the
// registers of eight, else two.
struct KeyPlan {
  int parts;       // of the line; 0: a workgroup an item
  int64_t items;   // at most
  int64_t slots;   // partial results that may be left: a part's place is its workgroup + its item
};
KeyPlan key_plan(int64_t rq, int64_t rk, int n, int kv, int per, int d, bool bf16) {
  const int blocks = (d + 31) / 32, keys = keys_of(bf16, blocks);
  const int64_t items = (rk / keys + 1 + n) * kv;
  if (rq * per <= 512) return {0, items, 0};
  const int parts = bf16 && keys == 64 ? 512 : 256;
  return {parts, items, parts + items};
}

template <typename E, int DB>
hipError_t run(const Args& A, bool token, hipStream_t st) {
  using T = typename std::conditional<std::is_same<E, float>::value, Split, E>::type;
  using L = Tile<T, DB>;
  constexpr int FLAGS = in_parts<T> ? kFlags : 0;
  if (A.index && (A.rq > 0 || A.rk > 0)) {
    hipLaunchKernelGGL((k_attn_index<KeySums<keys_of(sizeof(E) == 2, DB), sizeof(E) == 2>>), dim3(1), dim3(kIndexThreads), 0, st, A, (int64_t*)A.index);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (A.rq > 0 && token) {
    constexpr int PITCH = Tile<E, DB>::PITCH;
    hipLaunchKernelGGL((k_attn_dq_token<E, DB>), dim3(A.waves / 4), dim3(kThreads), 8 * kUnit * PITCH, st, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_attn_dq_join<E, DB>), flat_grid(A.rq * A.heads), dim3(kThreads), 0, st, A);
    const hipError_t f = hipGetLastError();
    if (f != hipSuccess) return f;
  } else if (A.rq > 0) {
    const int64_t tiles = (A.rq * A.per + kRows - 1) / kRows + A.n;
    if (!crowded<T>(DB) && split_keys(A, tiles))
      hipLaunchKernelGGL((k_attn_dq<T, (crowded<T>(DB) ? 1 : DB), 2>), flat_grid(tiles * A.kv), dim3(2 * kThreads), 8 * L::BYTES + FLAGS, st, A);
    else
      hipLaunchKernelGGL((k_attn_dq<T, DB, 1>), flat_grid(tiles * A.kv), dim3(kThreads), 4 * L::BYTES + FLAGS, st, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (A.rk > 0) {
    constexpr int KEYS = keys_of(sizeof(E) == 2, DB);
    const KeyPlan p = key_plan(A.rq, A.rk, A.n, A.kv, A.per, A.d, sizeof(E) == 2);
    Args B = A;
    B.waves = p.parts;
    B.slots = p.slots;
    hipLaunchKernelGGL((k_attn_dkv<T, DB>), flat_grid(p.parts ? p.parts : p.items), dim3(4 * KEYS),
                       2 * ((crowded<T>(DB) ? 0 : KEYS) + kQRows) * L::PITCH * L::PL + 2 * kQRows * 4 + FLAGS, st, B);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.parts) hipLaunchKernelGGL((k_attn_dkv_join<E, DB>), flat_grid(p.items, DB), dim3(4 * KEYS), 0, st, B);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t run_db(const Args& A, bool token, hipStream_t st) {
  switch ((A.d + 31) / 32) {
    case 1: return run<T, 1>(A, token, st);
    case 2: return run<T, 2>(A, token, st);
    case 3: return run<T, 3>(A, token, st);
    default: return run<T, 4>(A, token, st);
  }
}

}  // namespace

size_t backward_part_bytes(int64_t rq, int64_t rk, int n, int kv, int per, int d, bool bf16) {
  const int blocks = (d + 31) / 32;
  return rk > 0 ? (size_t)key_plan(rq, rk, n, kv, per, d, bf16).slots * 2 * keys_of(bf16, blocks) * blocks * 32 * sizeof(float) : 0;
}

hipError_t launch_backward(const Args& A, bool bf16, bool token, hipStream_t st) {
  return bf16 ? run_db<__bf16>(A, token, st) : run_db<float>(A, token, st);
}

}  // namespace attn
}  // namespace dnb
