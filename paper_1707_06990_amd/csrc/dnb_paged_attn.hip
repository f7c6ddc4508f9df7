// Attention of new tokens over a paged cache: softmax(scale q k^T) v for each sequence and head, the queries being a sequence's
// last tokens and the keys rows of pages that a table names.
//
// As in dnb_attn.hip the `per` query heads of a key/value head are rows of one matrix (packed row m is query m / per, head
// m % per of the group).  A workgroup of four waves takes a block of packed rows of one key/value head and walks over its keys
// in steps of KT.  A wave holds 32 rows: with many rows the four have 32 each and share all keys, with
// few they share the rows and each step's keys (KH waves to a set of rows).
// Batches mix single tokens over long caches with chunks of prompts, and only the device knows which: all (block, step)
// units lie on one line, in units of their cost, which is cut into equal parts, one a workgroup.  A block that several
// workgroups share leaves its sums, not yet divided, in the workspace, and k_paged_join adds them.
//
// What bounds it, at 32 heads over 8 of 128 in bf16 with pages of 16: single tokens the reading of the cache (21 of them over 78039
// keys, 320 MB: 72 us, 4.4 TB/s; of a large copy 5.05), chunks of prompts the issue of products and exponentials by the one wave a SIMD
// (4 x 1024 over 8192 keys: 515 to 563 us on different cards, 1001 to 915 TFLOP/s; a large product 1321), a lone token over 777 keys
// latency alone: 11 us of the first kernel's 13 are finding its part, the queries and the first keys, one after another, and 4 the join.  In fp32 six products of bf16
// parts stand for one (16 heads over 4 of 64, 4 x 1024 over 4096 keys: 408 us, 147 of 220 TFLOP/s): two workgroups a CU, 488 us with one.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>
#include <type_traits>

#include "dnb_attn_dev.h"
#include "dnb_paged.h"

namespace dnb {
namespace attn {
namespace {

constexpr int kThreads = 256;

// A block that workgroups share, as its first one leaves it for the join; parts 0: none.
struct Shared {
  int q0, m0, rows, g, parts;
};

struct PArgs {
  const void *q, *k, *v;
  void* o;
  float *lse, *part;
  Shared* shared;
  const int32_t *qo, *lens, *table;
  int n, heads, kv, per, d, causal, columns, shift, W;
  int64_t pages, rq, qs, ps, rs, hs;
  float c;  // scale * log2(e)
  uint32_t per_mul, per_shift;
  int cost[3], extra[3], least;  // see Blocks; the least that a workgroup is given
};

// m / per, m below 2^31
__device__ __forceinline__ int query_of(const PArgs& A, int m) { return A.per == 1 ? m : (int)(__umulhi((uint32_t)m, A.per_mul) >> A.per_shift); }

// 16 bytes of the tensors' zeros, twice: where rows that are not there are read
__device__ __attribute__((aligned(32))) const float kZeros[8] = {};

struct PSeq {
  int q0, nq, nk;
};
__device__ __forceinline__ PSeq pseq_at(const PArgs& A, int i) {
  PSeq s;
  const int64_t q0 = min(max((int64_t)A.qo[i], (int64_t)0), A.rq), q1 = min(max((int64_t)A.qo[i + 1], q0), A.rq);
  s.q0 = (int)q0;
  s.nq = (int)(q1 - q0);
  s.nk = (int)min((int64_t)max(A.lens[i], 0), (int64_t)A.columns << A.shift);
  return s;
}
__device__ __forceinline__ unsigned pseen(const PArgs& A, const PSeq& S, int m) {
  return A.causal ? max(S.nk + min(query_of(A, m) + 1 - S.nq, 0), 0) : S.nk;
}

// Blocks of a sequence: `rw` of the four waves take 32 * NC rows each, and with up to 32 rows one set of 32.  Their place on
// the line: `extra` units for the beginning and the end, then `cost` a step.
template <int KT, int NC>
struct Blocks {
  int rw, rows, count, cost, extra, M;
  __device__ __forceinline__ Blocks(const PArgs& A, const PSeq& S) {
    M = S.nq * A.per;
    const bool narrow = KT >= 128 && M <= 32;
    rw = narrow ? 1 : M <= 64 * NC ? 2 : 4;
    rows = narrow ? 32 : 32 * NC * rw;
    count = (M + rows - 1) / rows;
    cost = rw == 4 ? A.cost[2] : A.cost[rw - 1];
    extra = rw == 4 ? A.extra[2] : A.extra[rw - 1];
  }
  // (a block whose rows see nothing takes a step too: its results are written)
  __device__ __forceinline__ int steps(const PArgs& A, const PSeq& S, int t) const {
    return max((int)((pseen(A, S, min((t + 1) * rows, M) - 1) + KT - 1) / KT), 1);
  }
  __device__ __forceinline__ int64_t units(const PArgs& A, const PSeq& S, int t) const { return extra + (int64_t)steps(A, S, t) * cost; }
  // first step that begins x units from the block's start or later
  __device__ __forceinline__ int step_at(int64_t x) const { return x <= extra ? 0 : (int)((uint32_t)(x - extra) + cost - 1) / cost; }
};
// of one key/value head, by a lane alone
template <int KT, int NC>
__device__ __forceinline__ int64_t head_units(const PArgs& A, const PSeq& S) {
  const Blocks<KT, NC> B(A, S);
  int64_t u = 0;
  if (!A.causal) return (int64_t)B.count * (B.count > 0 ? B.units(A, S, 0) : 0);
  for (int t = 0; t < B.count; ++t) u += B.units(A, S, t);
  return u;
}

// Sum over the threads up to each; *total: over all.  `red`: room for four in LDS, free again after the caller's next barrier.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* red, int64_t* total) {
  const int wave = threadIdx.x >> 6;
  int64_t s = wave_scan(v);
  __syncthreads();
  if (lane_id() == 63) red[wave] = s;
  __syncthreads();
  int64_t all = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < wave) s += red[i];
    all += red[i];
  }
  *total = all;
  return s;
}

// A tile's rows on their way to LDS; rows of keys from key0 on, of which nk exist, as the table says where they lie.
template <typename T, int DB, int ROWS>
struct PagedStage {
  using L = Tile<T, DB>;
  using E = elem_t<T>;
  static constexpr int U = ROWS * L::CH / kThreads;
  static_assert(ROWS * L::CH % kThreads == 0, "");
  u32x4 k[U * L::LD], v[U * L::LD];
  __device__ __forceinline__ void load(const PArgs& A, const int32_t* table, int64_t head, int tid, unsigned key0, unsigned nk) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = tid + u * kThreads, row = i / L::CH, c = i - row * L::CH;
      const unsigned key = key0 + row;
      bool in = key < nk && c * L::EP < A.d;
      const int page = in ? table[key >> A.shift] : -1;
      in = page >= 0 && page < A.pages;
      const int64_t at = page * A.ps + (int64_t)(key & ((1u << A.shift) - 1)) * A.rs + head + c * L::EP;
      const E* kp = in ? (const E*)A.k + at : (const E*)kZeros;
      const E* vp = in ? (const E*)A.v + at : (const E*)kZeros;
#pragma unroll
      for (int p = 0; p < L::LD; ++p) {
        k[u * L::LD + p] = reinterpret_cast<const u32x4*>(kp)[p];
        v[u * L::LD + p] = reinterpret_cast<const u32x4*>(vp)[p];
      }
    }
  }
  __device__ __forceinline__ void store(lds_t kt, lds_t vt, int tid) {
    store_pieces<T, DB, U, kThreads, ROWS>(kt, tid, k);
    store_pieces<T, DB, U, kThreads, ROWS>(vt, tid, v);
  }
};

template <int DB>
constexpr int part_floats(int rows) { return rows * (32 * DB + 2); }

// Where a block's results go: the output, or a part's place.
struct Target {
  int q0, m0, M, g;
  float* part;  // null: the output
  int rows;     // of the part's place
};

// The KH waves of a set of rows join: O, m and l of waves kh > 0 through LDS (free, behind a barrier).
template <int DB>
__device__ __forceinline__ void join_waves(Online<DB>& R, char* shared, int wave, int KH) {
  const int l = lane_id(), kh = wave & (KH - 1);
  constexpr int PIECES = DB * 4 + 1;
  f32x4* to = reinterpret_cast<f32x4*>(shared) + wave * PIECES * 64 + l;
  if (kh > 0) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) to[(db * 4 + q) * 64] = (f32x4){R.o[db][4 * q], R.o[db][4 * q + 1], R.o[db][4 * q + 2], R.o[db][4 * q + 3]};
    to[DB * 4 * 64] = (f32x4){R.m, R.l, 0.f, 0.f};
  }
  __syncthreads();
  if (kh > 0) return;
  for (int w = 1; w < KH; ++w) {
    const f32x4* from = to + w * PIECES * 64;
    const f32x4 ml = from[DB * 4 * 64];
    const float m = fmaxf(R.m, ml[0]), t = m == -INFINITY ? 0.f : m;
    const float a = __builtin_amdgcn_exp2f(R.m - t), b = __builtin_amdgcn_exp2f(ml[0] - t);
    R.m = m;
    R.l = R.l * a + ml[1] * b;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 x = from[(db * 4 + q) * 64];
#pragma unroll
        for (int k = 0; k < 4; ++k) R.o[db][4 * q + k] = R.o[db][4 * q + k] * a + x[k] * b;
      }
  }
}

template <typename E, int DB>
__device__ __forceinline__ void write_rows(const PArgs& A, const Target& to, const f32x16 (&o)[DB], float top, float half, int row0) {
  const int l = lane_id(), r = row0 + (l & 31), m = to.m0 + r;
  const bool valid = m < to.M;
  const float sum = half_sum(half);
  if (to.part) {
    store_cols<float, DB>(to.part + (int64_t)r * 32 * DB, valid, 32 * DB, o, 1.f);
    if (valid && l < 32) {
      to.part[to.rows * 32 * DB + r] = top;
      to.part[to.rows * (32 * DB + 1) + r] = sum;
    }
    return;
  }
  const int query = query_of(A, m), head = to.g * A.per + m - query * A.per;
  const int64_t qrow = (int64_t)to.q0 + query;
  store_cols<E, DB>((E*)A.o + (qrow * A.heads + head) * A.d, valid, A.d, o, sum == 0.f ? 0.f : 1.f / sum);
  if (valid && l < 32 && A.lse) A.lse[(int64_t)head * A.rq + qrow] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

template <typename T, int DB>
struct Walk {
  static constexpr int KT = 64, NC = 1;
  using L = Tile<T, DB>;
  using E = elem_t<T>;
  static constexpr int TILE = KT * L::PITCH * L::PL;
  static constexpr int JOIN = 4 * (DB * 4 + 1) * 64 * 16;
  static constexpr int BYTES = (2 * TILE > JOIN ? 2 * TILE : JOIN) + kFlags;

  // Steps first .. last - 1 of a block.
  static __device__ __forceinline__ void run(const PArgs& A, char* shared, const PSeq& S, const int32_t* table, const Blocks<KT, NC>& B, int g,
                                             int t, int first, int last, const Target& to) {
    const lds_t lds = lds_start(shared);
    const int wave = threadIdx.x >> 6, l = lane_id(), KH = 4 / B.rw, kh = wave & (KH - 1), row0 = wave / KH * 32;
    const int m = t * B.rows + row0 + (l & 31), query = query_of(A, m), head = g * A.per + m - query * A.per;
    const bool valid = m < B.M;
    const unsigned sees = pseen(A, S, m);
    const int m0 = t * B.rows + row0;
    const unsigned most = m0 >= B.M ? 0 : pseen(A, S, min(m0 + 31, B.M - 1)), least = pseen(A, S, m0);
    const unsigned all = pseen(A, S, min((t + 1) * B.rows, B.M) - 1);  // keys that the block's last row sees
    const int blocks = KT / 32 / KH;
    Online<DB> R;
    auto walk = [&](auto form) {
      using F = decltype(form);
      Columns<F, DB> qf;
      load_cols<F, DB>(qf, (const E*)A.q + ((int64_t)S.q0 + apart<F>(query)) * A.qs + (int64_t)apart<F>(head) * A.d, valid, A.d);
      R.init();
      PagedStage<F, DB, KT> stage;
      const int tid = apart<F>((int)threadIdx.x);
      if (!is_whole<F> && first < last) stage.load(A, table, g * A.hs, tid, first * KT, all);
      for (int s = first; s < last; ++s) {
        if (is_whole<F>) stage.load(A, table, g * A.hs, tid, s * KT, all);
        __syncthreads();
        stage.store(lds, lds + TILE, tid);
        __syncthreads();
        if (!is_whole<F> && s + 1 < last) stage.load(A, table, g * A.hs, tid, (s + 1) * KT, all);
        for (int b = 0; b < blocks; ++b) {
          const int r = (kh * blocks + b) * 32;
          const unsigned key = (unsigned)s * KT + r;
          if (key >= most) break;
          f32x16 x[1] = {row_mul<F, DB, false, KT>(lds, r, qf)};
          if (key + 32 > least) hide(x[0], key, sees);
          online_step<F, DB, 1, false, KT>(R, x, A.c, lds + TILE, r);
        }
      }
    };
    walk(T());
    if constexpr (L::PL == 3) {
      __syncthreads();
      if (any_wave<4>(lds + BYTES - kFlags, not_finite(R.o))) walk(Whole());
    }
    if (KH > 1) {
      __syncthreads();
      join_waves<DB>(R, shared, wave, KH);
    }
    if (kh == 0) write_rows<E, DB>(A, to, R.o, R.m, R.l, row0);
  }
};

// ---------------------------------------------------------------- bf16

// O, maximum and sum of N sets of 32 rows.
template <int DB, int N>
struct Sets {
  f32x16 o[N][DB];
  float m[N], l[N];
};

// Keys and values of a step on their way from the pages to LDS, without passing through registers: a load instruction of
// a wave fills 1 KB of LDS, RPI rows, lane after lane; which piece of its row a lane fetches is turned round so that the tile's
// order comes out.  The wave has rows wave * 32 .. + 31, U instructions for K and as many for V.  Where its groups of RPI rows begin
// is computed for WINDOW steps at once, a group a lane.
template <int DB>
struct Fetch {
  using L = Tile<__bf16, DB>;
  static constexpr int RPI = 64 / L::PC, U = 32 / RPI, WINDOW = 64 / U;
  uint64_t from;      // lane i: the first key row of step base + i / U, group i % U
  int64_t apart_by;   // from a key's bytes to its value's
  int clean;          // all pages of the window, of all waves, are of the pool
  int base;           // the window's first step
  int next;           // the following window's pages
  int next_clean;
  uint32_t row_at, c16;  // bytes from a group's first row to the lane's; the lane's piece in group 0
  const int32_t* table;
  int64_t head;       // bytes

  __device__ __forceinline__ unsigned key_of(int step, int wave) const {
    const int l = lane_id();
    return (unsigned)(step + l / U) * 128u + wave * 32u + (l % U) * RPI;
  }
  __device__ __forceinline__ void look(const PArgs& A, int step, unsigned nk) {
    bool in = true;
    const int mine = threadIdx.x >> 6;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const unsigned key = key_of(step, w);
      const int page = key < nk ? table[key >> A.shift] : 0;
      in = in && (unsigned)page < A.pages;
      if (w == mine) next = page;
    }
    next_clean = __ballot(!in) == 0;
  }
  __device__ __forceinline__ void place(const PArgs& A) {
    from = (uint64_t)A.k + head + (uint64_t)(uint32_t)next * (uint32_t)(A.ps * 2) +
           (uint64_t)(key_of(base, threadIdx.x >> 6) & ((1u << A.shift) - 1)) * (uint32_t)(A.rs * 2);
    clean = next_clean;
  }
  __device__ __forceinline__ void init(const PArgs& A, const int32_t* t, int g, int first, unsigned nk) {
    const int l = lane_id();
    table = t;
    head = (int64_t)g * A.hs * 2;
    apart_by = (const char*)A.v - (const char*)A.k;
    base = first;
    row_at = (uint32_t)(l / L::PC) * (uint32_t)(A.rs * 2);
    c16 = (uint32_t)((l % L::PC) ^ L::swz(l / L::PC)) * 16;
    look(A, first, nk);
    place(A);
    look(A, first + WINDOW, nk);
  }
  __device__ __forceinline__ void turn(const PArgs& A, int step, unsigned nk) {
    if (step < base + WINDOW) return;
    base += WINDOW;
    place(A);
    look(A, base + WINDOW, nk);
  }
  // A group of keys and its values.  `from` comes out of v_readlane, and a memory instruction must not take its address from scalar
  // registers within five wait states of a vector instruction that writes them: one for s_mov, four for s_nop 3 (the compiler does not
  // count for instructions that it does not know).  m0 needs one.  Both loads in one block, so that the second has waited too (four
  // chunks 440 us; 449 with the wait before each).
  static __device__ __forceinline__ void load(lds_t kt, lds_t vt, uint32_t voff, uint64_t k, uint64_t v) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %4"
                 ::"s"(__builtin_amdgcn_readfirstlane(kt)), "s"(__builtin_amdgcn_readfirstlane(vt)), "v"(voff), "s"(k), "s"(v) : "memory", "m0");
  }
  static __device__ __forceinline__ void load(lds_t to, const char* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "memory", "m0");
  }
  // Whether all rows of a step (of this window) are there, with as many pieces as a tile's, in groups within a page and with
  // offsets of 32 bits.  The same for all waves.
  __device__ __forceinline__ bool quick(const PArgs& A, int step, unsigned nk) const {
    return clean && ((unsigned)step + 1) * 128u <= nk && A.d == 32 * DB && (1 << A.shift) >= RPI && A.rs < (1 << 26);
  }
  // Group u of such a step; kt, vt: of the wave's rows.
  __device__ __forceinline__ void group(lds_t kt, lds_t vt, int step, int u) const {
    const int i = (step - base) * U + u;
    const uint64_t f = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(from >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)from, i);
    uint32_t c = c16 ^ (uint32_t)(L::swz(u * RPI) * 16);
    if (L::CH < L::PC) c = min(c, (uint32_t)(L::CH - 1) * 16);  // (pieces past a row's are not read)
    load(kt + u * 1024, vt + u * 1024, row_at + c, f, f + apart_by);
  }
  // Step `step` into the tiles at kt and vt; nk: keys that exist.
  __device__ __forceinline__ void issue(const PArgs& A, lds_t kt, lds_t vt, int step, unsigned nk) const {
    const int l = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    kt += wave * 32 * L::PITCH;
    vt += wave * 32 * L::PITCH;
    if (quick(A, step, nk)) {
#pragma unroll 2
      for (int u = 0; u < U; ++u) group(kt, vt, step, u);
      return;
    }
    // What is not there comes from the zeros.  (The lookups all before the first load into LDS, for which a later one would wait.)
    const unsigned key0 = (unsigned)step * 128u + wave * 32u, mask = (1u << A.shift) - 1;
    int pages[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const unsigned key = key0 + u * RPI + l / L::PC;
      pages[u] = key < nk ? table[key >> A.shift] : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" ::"v"(pages[u]));
    const char* k = (const char*)A.k + head;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const unsigned key = key0 + u * RPI + l / L::PC;
      const int c = (l % L::PC) ^ L::swz(l / L::PC) ^ L::swz(u * RPI);
      const bool in = key < nk && c * 8 < A.d && (unsigned)pages[u] < A.pages;
      const char* p = k + (uint64_t)(uint32_t)pages[u] * (uint32_t)(A.ps * 2) + (uint64_t)(key & mask) * (uint32_t)(A.rs * 2) + c * 16;
      load(kt + u * 1024, in ? p : (const char*)kZeros);
      load(vt + u * 1024, in ? p + apart_by : (const char*)kZeros);
    }
  }
};

template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int DB>
struct Walk<__bf16, DB> {
  static constexpr int KT = 128, NC = 2;
  using L = Tile<__bf16, DB>;
  using F = Fetch<DB>;
  static constexpr int TILE = KT * L::PITCH;
  static constexpr int JOIN = 256 * (32 * DB + 2) * 4;
  static constexpr int BYTES = (4 * TILE > JOIN ? 4 * TILE : JOIN) + kFlags;

  template <int N>
  using Scores = f32x16[N];
  template <int N>
  using Queries = Piece[N][L::NS][1];

  template <int N>
  static __device__ __forceinline__ void scores(Scores<N>& s, const Queries<N>& q, lds_t at) {
#pragma unroll
    for (int n = 0; n < N; ++n) s[n] = (f32x16){};
#pragma unroll
    for (int k = 0; k < L::NS; ++k) {
      Piece a[1];
      a[0].q = lds_read<u32x4>(at ^ (k << 5));
#pragma unroll
      for (int n = 0; n < N; ++n) mma(s[n], a, q[n][k], (__bf16*)nullptr);
    }
  }
  template <int N>
  static __device__ __forceinline__ void values(Sets<DB, N>& R, const Scores<N>& s, lds_t at) {
    using lds4 = __attribute__((address_space(3))) s16x4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      Piece y[N][1];
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int j = 0; j < 8; ++j) y[n][0].b[j] = (__bf16)s[n][8 * t + j];
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        Piece x[1];
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(uintptr_t)((at ^ (db << 6)) + 16 * t * L::PITCH));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(uintptr_t)((at ^ (db << 6) ^ 32) + (16 * t + 8) * L::PITCH));
        const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
        x[0].q = (u32x4){a.x, a.y, b.x, b.y};
#pragma unroll
        for (int n = 0; n < N; ++n) mma(R.o[n][db], x, y[n], (__bf16*)nullptr);
      }
    }
  }
  // Largest raw score of each column
  template <int N>
  static __device__ __forceinline__ void tops(float (&top)[N], const Scores<N>& s) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float t = s[n][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) t = fmaxf(t, s[n][i]);
      top[n] = half_max(t);
    }
  }
  // The sums so far take the new maximum where it has grown by more than 8 (a factor of 256).
  template <int N>
  static __device__ __forceinline__ void rescale(Sets<DB, N>& R, float (&top)[N], float c) {
    bool grow = false;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      top[n] *= c;  // c > 0
      grow |= top[n] > R.m[n] + 8.f;  // (-inf + 8 is -inf: so is the first that is more)
    }
    if (__builtin_expect_with_probability(!__any(grow), 1, 0.999)) return;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float m = fmaxf(R.m[n], top[n]);
      const float a = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(R.m[n] - m);
      R.m[n] = m;
      R.l[n] *= a;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
#pragma unroll
        for (int i = 0; i < 16; ++i) R.o[n][db][i] *= a;
      }
    }
  }
  template <int N>
  static __device__ __forceinline__ void weights(Sets<DB, N>& R, Scores<N>& s, float c) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float m = R.m[n] == -INFINITY ? 0.f : R.m[n];
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], c, -m));
        t += s[n][i];
      }
      R.l[n] += t;
    }
  }

  // A block of 32 keys, whose scores are s, and beside it the scores of the following one: a product's 32 cycles are another
  // seven instructions' time.  There is one wave a SIMD, so what it waits for is lost: reads of LDS go out three phases (of N
  // products) before their use, and every product has its share of the other instructions behind it, which stay there.
  // The maximum is that of the first block, R.m, for all: weights have the exponents of fp32, and are as exact at 2^60 as at 1;
  // sums that have left their range are seen at the end, and the work is done again with a running maximum (see odd and again).
  // A row's sum is that of its weights before they are rounded to bf16, one after another.
  // load(k): something more for phase k, of the first.
  // HIDE: keys of the following block from next_key on, of which a lane's rows see those below sees.
  template <int N, bool HIDE, typename Load>
  static __device__ __forceinline__ void block(Sets<DB, N>& R, Scores<N>& s, Scores<N>& sn, const float (&minus)[N],
                                               const Queries<N>& q, float c, lds_t k_at, lds_t v_at, Load load,
                                               unsigned next_key = 0, const unsigned* sees = nullptr) {
    constexpr int NS = L::NS, NV = 2 * DB, AHEAD = 3;
    Piece f[NS + NV][1];
    auto read = [&](int i) {
      if (i < NS) {
        f[i][0].q = lds_read<u32x4>(k_at ^ (i << 5));
      } else if (i < NS + NV) {
        using lds4 = __attribute__((address_space(3))) s16x4;
        const int t = (i - NS) / DB, db = (i - NS) % DB;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(uintptr_t)((v_at ^ (db << 6)) + 16 * t * L::PITCH));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(uintptr_t)((v_at ^ (db << 6) ^ 32) + (16 * t + 8) * L::PITCH));
        const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
        f[i][0].q = (u32x4){a.x, a.y, b.x, b.y};
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read(i);
    Piece y[2][N][1];
    float p[2][N][8];
#pragma unroll
    for (int n = 0; n < N; ++n) sn[n] = (f32x16){};
    // The weights in the order in which the products need them, spread over the time until the last do.
    constexpr int SPOTS = (NS + DB) * N, REST = DB * N;
#pragma unroll
    for (int i = 0; i < NS + NV; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int spot = i * N + n;
        if (n == 0) read(i + AHEAD);
        if (i < NS) mma(sn[n], f[i], q[n][i], (__bf16*)nullptr);
        else mma(R.o[n][(i - NS) % DB], f[i], y[(i - NS) / DB][n], (__bf16*)nullptr);
        if (i < NS && n == 0) load(i);
        asm volatile("" : "+s"(c));  // the weights that follow here, and not together with others
#pragma unroll
        for (int e = 0; e < 16 * N; ++e) {
          const int t = e / (8 * N), col = e / 8 % N, j = e % 8, at = e * (SPOTS - 2) / (16 * N);
          float& x = p[t][col][j];
          if (at == spot) x = fmaf(s[col][8 * t + j], c, minus[col]);
          if (at + 1 == spot) {
            asm volatile("" : "+v"(x));
            x = __builtin_amdgcn_exp2f(x);
          }
          if (at + 2 == spot) {
            asm volatile("" : "+v"(x));
            R.l[col] += x;
            y[t][col][0].b[j] = (__bf16)x;
          }
        }
        if (HIDE) {
#pragma unroll
          for (int e = 0; e < 16 * N; ++e)
            if (SPOTS + e * REST / (16 * N) == spot) {
              const int col = e / 16, j = e % 16;
              sn[col][j] = next_key + row_of(j) >= sees[col] ? -INFINITY : sn[col][j];
            }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
  }
  // The first block's scores: the maximum for all.
  template <int N>
  static __device__ __forceinline__ void settle(Sets<DB, N>& R, const Scores<N>& s, float c, float (&minus)[N]) {
    float top[N];
    tops<N>(top, s);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      R.m[n] = top[n] * c;
      // (where the first block has nothing, nor must later ones: any score above -inf makes an infinite weight)
      minus[n] = R.m[n] == -INFINITY ? 3.4e38f : -R.m[n];
    }
  }
  template <int N>
  static __device__ __forceinline__ void clear(Sets<DB, N>& R) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
      for (int db = 0; db < DB; ++db) R.o[n][db] = (f32x16){};
      R.m[n] = -INFINITY;
      R.l[n] = 0.f;
    }
  }
  // Sums that scores far above the first block's have made large, so large that parts of a row could not be added, or that
  // are not finite, in any of the wave's rows.
  template <int N>
  static __device__ __forceinline__ bool odd(const Sets<DB, N>& R) {
    bool b = false;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float most = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(R.o[n][db][i]));
      b = b | !(R.l[n] < 0x1p64f) | (most > 0x1p100f) | not_finite(R.o[n]);
    }
    return __any(b);
  }

  // The KH waves of a set of rows join, and the results go where they belong.  Each wave's sums go to LDS, a row after
  // another, 16-byte pieces turned round by the row against bank conflicts; then a thread takes four values of a row.
  template <int N>
  static __device__ __forceinline__ void join(const PArgs& A, char* shared, const Sets<DB, N>& R, const Blocks<KT, NC>& B, const Target& to) {
    constexpr int PIECES = 8 * DB, DP = 32 * DB;
    const int wave = threadIdx.x >> 6, l = lane_id(), KH = 4 / B.rw;
    f32x4* o = reinterpret_cast<f32x4*>(shared);                           // (wave, row, piece)
    float2* ml = reinterpret_cast<float2*>(shared + 128 * N * DP * 4);  // (wave, row)
    const int rows = min(B.rows, to.M - to.m0);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int r = 32 * n + (l & 31), slot = wave * 32 * N + r;
      const float sum = half_sum(R.l[n]);
      if (wave / KH * 32 * N + r < rows) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            o[slot * PIECES + ((8 * db + 2 * g + (l >> 5)) ^ (r & 7))] = (f32x4){R.o[n][db][4 * g], R.o[n][db][4 * g + 1], R.o[n][db][4 * g + 2], R.o[n][db][4 * g + 3]};
        if (l < 32) ml[slot] = make_float2(R.m[n], sum);
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < rows * PIECES; e += kThreads) {
      const int row = e / PIECES, c = e - row * PIECES, r = row % (32 * N), slot = row / (32 * N) * KH * 32 * N + r;
      float m = -INFINITY, sum = 0.f;
      for (int k = 0; k < KH; ++k) m = fmaxf(m, ml[slot + k * 32 * N].x);
      const float z = m == -INFINITY ? 0.f : m;
      f32x4 y = {};
      for (int k = 0; k < KH; ++k) {
        const float2 x = ml[slot + k * 32 * N];
        const float f = __builtin_amdgcn_exp2f(x.x - z);
        const f32x4 v = o[(slot + k * 32 * N) * PIECES + (c ^ (r & 7))];
        sum = fmaf(x.y, f, sum);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = fmaf(v[j], f, y[j]);
      }
      const int mm = to.m0 + row;
      if (to.part) {
        *reinterpret_cast<f32x4*>(to.part + (int64_t)row * DP + 4 * c) = y;
        if (c == 0) {
          to.part[to.rows * DP + row] = m;
          to.part[to.rows * (DP + 1) + row] = sum;
        }
        continue;
      }
      const int query = query_of(A, mm), head = to.g * A.per + mm - query * A.per;
      const int64_t qrow = (int64_t)to.q0 + query;
      if (4 * c < A.d) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<bf16x4*>((__bf16*)A.o + (qrow * A.heads + head) * A.d + 4 * c) = (bf16x4){(__bf16)(y[0] * f), (__bf16)(y[1] * f), (__bf16)(y[2] * f), (__bf16)(y[3] * f)};
      }
      if (c == 0 && A.lse) A.lse[(int64_t)head * A.rq + qrow] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
    }
  }

  // The wave's N sets of 32 rows from row m0 of the matrix on
  template <int N>
  static __device__ __forceinline__ void begin(const PArgs& A, const PSeq& S, const Blocks<KT, NC>& B, int g, int m0, Queries<N>& q, unsigned (&sees)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int m = m0 + 32 * n + (lane_id() & 31), query = query_of(A, m), head = g * A.per + m - query * A.per;
      sees[n] = pseen(A, S, m);
      load_cols<__bf16, DB>(q[n], (const __bf16*)A.q + ((int64_t)S.q0 + query) * A.qs + (int64_t)head * A.d, m < B.M, A.d);
    }
  }
  static __device__ __forceinline__ lds_t k_lane() { return L::at(lane_id() & 31, lane_id() >> 5); }
  static __device__ __forceinline__ lds_t v_lane() {
    const int l = lane_id();
    return L::at(4 * (l >> 5) + ((l >> 2) & 3), 2 * ((l >> 4) & 1) + ((l >> 1) & 1)) + (l & 1) * 8;
  }
  // The steps with a running maximum, for scores that leave the first block's far behind, and sums that are not finite: one after
  // another, all four waves together.  Where nearly every part has to, 4 x 1024 over 8192 keys take 1213 us for 539, 21 single
  // tokens over 78039 keys 127 for 72, 64 over 1024 keys each 95 for 64.
  template <int N>
  static __device__ __forceinline__ void again(const PArgs& A, F& f, lds_t kt, lds_t vt, int g, int first, int last, unsigned all, int nb, int kh,
                                               const Queries<N>& q, const unsigned (&sees)[N], Sets<DB, N>& R) {
    clear<N>(R);
    f.init(A, f.table, g, first, all);
#pragma unroll 1
    for (int s = first; s < last; ++s) {
      __syncthreads();
      f.turn(A, s, all);
      f.issue(A, kt, vt, s, all);
      wait_loads<0>();
      __syncthreads();
#pragma unroll 1
      for (int j = 0; j < nb; ++j) {
        const int r = (kh * nb + j) * 32;
        Scores<N> a;
        float top[N];
        scores<N>(a, q, kt + k_lane() + r * L::PITCH);
#pragma unroll
        for (int n = 0; n < N; ++n) hide(a[n], (unsigned)s * KT + r, sees[n]);
        tops<N>(top, a);
        rescale<N>(R, top, A.c);
        weights<N>(R, a, A.c);
        values<N>(R, a, vt + v_lane() + r * L::PITCH);
      }
    }
  }

  // Up to 32 rows: each wave takes a fourth of every step's keys, which it fetches itself two steps ahead, and waits for nobody.
  static __device__ __forceinline__ void run_narrow(const PArgs& A, char* shared, const PSeq& S, const int32_t* table, const Blocks<KT, NC>& B, int g,
                                                    int first, int last, const Target& to) {
    const lds_t kt = lds_start(shared), vt = kt + 2 * TILE;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned all = pseen(A, S, B.M - 1), least = pseen(A, S, 0);
    F f;
    if (first < last) f.init(A, table, g, first, all);
    Queries<1> q;
    Sets<DB, 1> R;
    unsigned sees[1];
    begin<1>(A, S, B, g, 0, q, sees);
    clear<1>(R);
    const lds_t k_at = kt + k_lane() + wave * 32 * L::PITCH, v_at = vt + v_lane() + wave * 32 * L::PITCH;
    float minus[1] = {0.f};
#pragma unroll 1
    for (int s = first - 2; s < last; ++s) {
      const lds_t buf = (s - first) & 1 ? TILE : 0;
      if (s >= first) {
        if (s + 1 < last) wait_loads<2 * F::U>();
        else wait_loads<0>();
        Scores<1> a;
        scores<1>(a, q, k_at + buf);
        const unsigned key = (unsigned)s * KT + wave * 32;
        if (key + 32 > least) {
          asm volatile("");  // a branch, not selections in every step
          hide(a[0], key, sees[0]);
        }
        if (s == first) settle<1>(R, a, A.c, minus);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          a[0][i] = __builtin_amdgcn_exp2f(fmaf(a[0][i], A.c, minus[0]));
          sum += a[0][i];
        }
        R.l[0] += sum;
        values<1>(R, a, v_at + buf);
        wait_lds();
      }
      if (s + 2 < last) {
        f.turn(A, s + 2, all);
        f.issue(A, kt + buf, vt + buf, s + 2, all);
      }
    }
    if (any_wave<4>(kt + BYTES - kFlags, odd<1>(R))) again<1>(A, f, kt, vt, g, first, last, all, 1, wave, q, sees, R);
    join<1>(A, shared, R, B, to);
  }

  // More rows: N sets a wave, two or four waves side by side, and KH of them at the same rows.
  static __device__ __forceinline__ void run_wide(const PArgs& A, char* shared, const PSeq& S, const int32_t* table, const Blocks<KT, NC>& B, int g, int t,
                                                  int first, int last, const Target& to) {
    constexpr int N = NC;
    const lds_t kt = lds_start(shared), vt = kt + 2 * TILE;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), KH = 4 / B.rw, kh = wave & (KH - 1), row0 = wave / KH * 32 * N;
    const int nb = 4 / KH;  // blocks of 32 keys of this wave in a step
    const unsigned all = pseen(A, S, min((t + 1) * B.rows, B.M) - 1);  // keys that the block's last row sees
    // keys that all rows of the workgroup see: by that the waves choose their way, all the same one, between barriers
    const unsigned lowest = pseen(A, S, t * B.rows);
    F f;
    if (first < last) f.init(A, table, g, first, all);
    Queries<N> q;
    Sets<DB, N> R;
    unsigned sees[N];
    begin<N>(A, S, B, g, t * B.rows + row0, q, sees);
    clear<N>(R);
    if (first < last) {
      f.issue(A, kt, vt, first, all);
      wait_loads<0>();
      meet();
      const lds_t k_at0 = kt + k_lane() + kh * nb * 32 * L::PITCH, v_at0 = vt + v_lane() + kh * nb * 32 * L::PITCH;
      lds_t buf = 0;  // of the step at hand
      Scores<N> a, b;
      float minus[N];
      scores<N>(a, q, k_at0);
#pragma unroll
      for (int n = 0; n < N; ++n) hide(a[n], (unsigned)first * KT + kh * nb * 32, sees[n]);
      settle<N>(R, a, A.c, minus);
      int s = first;
      auto nothing = [](int) {};
      // Steps after which another comes and all of whose keys, and the next one's first, all rows see.  The next step's rows are
      // fetched group by group beside the products of the first two of four blocks.
      if (nb == 4) {
#pragma unroll 1
        for (; s + 1 < last && ((unsigned)s + 2) * KT <= lowest; ++s) {
          f.turn(A, s + 1, all);
          if (!f.quick(A, s + 1, all)) break;
          const lds_t k_at = k_at0 + buf, v_at = v_at0 + buf;
          const lds_t kw = kt + (buf ^ TILE) + wave * 32 * L::PITCH, vw = vt + (buf ^ TILE) + wave * 32 * L::PITCH;
          block<N, false>(R, a, b, minus, q, A.c, k_at + 32 * L::PITCH, v_at, [&](int k) { if (k < F::U / 2) f.group(kw, vw, s + 1, k); });
          block<N, false>(R, b, a, minus, q, A.c, k_at + 64 * L::PITCH, v_at + 32 * L::PITCH,
                          [&](int k) { if (k < F::U / 2) f.group(kw, vw, s + 1, F::U / 2 + k); });
          block<N, false>(R, a, b, minus, q, A.c, k_at + 96 * L::PITCH, v_at + 64 * L::PITCH, nothing);
          buf ^= TILE;
          // the next step is here
          wait_loads<0>();
          meet();
          block<N, false>(R, b, a, minus, q, A.c, k_at0 + buf, v_at + 96 * L::PITCH, nothing);
          // all have read this one
          wait_lds();
          meet();
        }
      }
      // The others.  (Blocks in one loop: loops of steps and blocks inside each other would copy all sums from one's registers to the
      // other's.)
      int j = 0;
#pragma unroll 1
      while (s < last) {
        const bool ends = j + 1 == nb, more = s + 1 < last;
        if (j == 0 && more) {
          f.turn(A, s + 1, all);
          f.issue(A, kt + (buf ^ TILE), vt + (buf ^ TILE), s + 1, all);
        }
        if (ends && more) {  // the next step is here
          wait_loads<0>();
          meet();
        }
        // (after the last block: scores of what lies there, all hidden)
        const lds_t next = ends ? k_at0 + (buf ^ TILE) : k_at0 + buf + (j + 1) * 32 * L::PITCH;
        const unsigned key = !ends ? (unsigned)s * KT + (kh * nb + j + 1) * 32 : more ? (unsigned)(s + 1) * KT + kh * nb * 32 : 0x80000000u;
        block<N, true>(R, a, b, minus, q, A.c, next, v_at0 + buf + j * 32 * L::PITCH, nothing, key, sees);
#pragma unroll
        for (int n = 0; n < N; ++n) a[n] = b[n];
        ++j;
        if (!ends) continue;
        j = 0;
        buf ^= TILE;
        ++s;
        // all have read this one
        wait_lds();
        meet();
      }
      if (any_wave<4>(kt + BYTES - kFlags, odd<N>(R))) again<N>(A, f, kt, vt, g, first, last, all, nb, kh, q, sees, R);
    }
    if (KH > 1) {
      join<N>(A, shared, R, B, to);
      return;
    }
#pragma unroll
    for (int n = 0; n < N; ++n) write_rows<__bf16, DB>(A, to, R.o[n], R.m[n], R.l[n], row0 + 32 * n);
  }
  static __device__ __forceinline__ void run(const PArgs& A, char* shared, const PSeq& S, const int32_t* table, const Blocks<KT, NC>& B, int g, int t,
                                             int first, int last, const Target& to) {
    if (B.rw == 1) run_narrow(A, shared, S, table, B, g, first, last, to);
    else run_wide(A, shared, S, table, B, g, t, first, last, to);
  }
};

// In fp32 with heads of up to 64 two workgroups a CU take turns at converting and multiplying (64 tokens over 1024 keys 61 -> 48 us); in
// bf16 one has all registers and 133 KB of LDS.
template <typename T, int DB>
__global__ __launch_bounds__(kThreads, (std::is_same<T, __bf16>::value || DB > 2 ? 1 : 2)) void k_paged(PArgs A, int max_rows) {
  using K = Walk<T, DB>;
  constexpr int KT = K::KT, NC = K::NC;
  using B_ = Blocks<KT, NC>;
  extern __shared__ __attribute__((aligned(512))) char shared[];
  int64_t* red = reinterpret_cast<int64_t*>(shared);
  const int tid = threadIdx.x, l = lane_id();
  int64_t mine = 0, first_units = 0, total;
  for (int i = tid; i < A.n; i += kThreads) {
    const int64_t u = head_units<KT, NC>(A, pseq_at(A, i)) * A.kv;
    if (i < kThreads) first_units = u;
    mine += u;
  }
  const int64_t scan = block_scan(mine, red, &total);
  const int W = (int)fmin((double)A.W, fmax((double)total / A.least, 1.0));
  // workgroups that lie side by side on the line run on one XCD, whose cache has the keys that they share
  const int w = A.W % 8 == 0 ? (int)(blockIdx.x % 8) * (A.W / 8) + (int)blockIdx.x / 8 : (int)blockIdx.x;
  if (tid == 0) A.shared[w].parts = 0;
  if (w >= W || total == 0) return;
  // parts of the line: total * w / W.  (In doubles: total is below 2^53 and W at most 512, so that quotients are right.)
  const int64_t share = (int64_t)((double)total / W), rest = total - share * W;
  const int64_t a = w * share + (int)(w * rest) / W, b = (w + 1) * share + (int)((w + 1) * rest) / W;
  // the sequence at a, and where on the line it begins
  int64_t* found = red + 4;
  int64_t before = 0;
  for (int base = 0; base < A.n; base += kThreads) {
    const int64_t u = A.n <= kThreads ? first_units : base + tid < A.n ? head_units<KT, NC>(A, pseq_at(A, base + tid)) * A.kv : 0;
    int64_t chunk = total;
    const int64_t end = before + (A.n <= kThreads ? scan : block_scan(u, red, &chunk));
    if (end > a && end - u <= a) {
      found[0] = base + tid;
      found[1] = end - u;
    }
    before += chunk;
    if (before > a) break;
  }
  __syncthreads();
  int i = __builtin_amdgcn_readfirstlane((int)found[0]);
  int64_t a0 = bcast64(found[1], 0);
  PSeq S = pseq_at(A, i);
  S = {bcast(S.q0, 0), bcast(S.nq, 0), bcast(S.nk, 0)};
  int g = 0, t = 0;
  {
    const B_ B(A, S);
    // key/value head and block at a
    if (B.count == 1) {
      const int64_t H = B.units(A, S, 0);
      g = (int)((double)(a - a0) / (double)H);
      a0 += g * H;
    } else {
      int64_t H = 0;
      for (int t0 = 0; t0 < B.count; t0 += 64) H += bcast64(wave_scan(t0 + l < B.count ? B.units(A, S, t0 + l) : 0), 63);
      g = (int)((double)(a - a0) / (double)H);
      a0 += g * H;
      for (int t0 = 0; t0 < B.count; t0 += 64) {
        const int64_t v = t0 + l < B.count ? B.units(A, S, t0 + l) : 0, end = a0 + wave_scan(v);
        const uint64_t past = __ballot(end > a);
        if (past) {
          const int at = __builtin_ctzll(past);
          t = t0 + at;
          a0 = bcast64(end - v, at);
          break;
        }
        a0 = bcast64(end, 63);
      }
    }
  }
  for (;;) {
    const B_ B(A, S);
    const int steps = B.steps(A, S, t);
    const int64_t a1 = a0 + B.extra + (int64_t)steps * B.cost;
    // a step is the workgroup's in whose part of the line it begins
    const int first = a0 < a ? B.step_at(a - a0) : 0, last = a1 > b ? min(steps, B.step_at(b - a0)) : steps;
    Target to = {S.q0, t * B.rows, B.M, g, nullptr, max_rows};
    if (a0 < a || a1 > b) {
      to.part = A.part + (int64_t)(2 * w + (a0 < a ? 0 : 1)) * part_floats<DB>(max_rows);
      if (a0 >= a && tid == 0) {
        // the last part's workgroup is the one with a1 - 1
        int e = max(w + 1, (int)((double)a1 / (double)total * W) - 2);
        while ((e + 1) * share + (int)((e + 1) * rest) / W < a1) ++e;
        A.shared[w] = {S.q0, t * B.rows, min(B.rows, B.M - t * B.rows), g, e - w + 1};
      }
    }
    __syncthreads();
    K::run(A, shared, S, A.table + (int64_t)i * A.columns, B, g, t, first, last, to);
    if (a1 >= b) return;
    a0 = a1;
    if (++t < B.count) continue;
    t = 0;
    if (++g < A.kv) continue;
    g = 0;
    for (++i; i < A.n; i += 64) {  // the next sequence that has rows
      const uint64_t some = __ballot(i + l < A.n && pseq_at(A, min(i + l, A.n - 1)).nq > 0);
      if (some) {
        i += __builtin_ctzll(some);
        break;
      }
    }
    if (i >= A.n) return;
    S = pseq_at(A, i);
    S = {bcast(S.q0, 0), bcast(S.nq, 0), bcast(S.nk, 0)};
  }
}

// Adds the parts of a shared block: 32 lanes (at head_dim 128) hold a row, and as many such groups as there are parts, up
// to all, take a row's parts side by side.  Workgroup (w, y): rows of the block that begins in workgroup w's part.
template <typename T, int DB>
__global__ __launch_bounds__(kThreads) void k_paged_join(PArgs A, int max_rows) {
  constexpr int DP = 32 * DB, LANES = DP / 4 > 16 ? 32 : DP / 4 > 8 ? 16 : 8, G = kThreads / LANES;
  __shared__ float red[G][DP + 2];
  const int w = blockIdx.x;
  const Shared S = A.shared[w];
  if (S.parts == 0) return;
  int split = 1;  // groups to a row: where there are few rows
  while (split < S.parts && split < G && S.rows * 2 * split <= (int)gridDim.y * G) split *= 2;
  const int grp = threadIdx.x / LANES, c = threadIdx.x % LANES, at = grp % split, rows = G / split;
  if (split == 1) {  // four rows a group at once, for loads in flight
    constexpr int R = 4;
    for (int r0 = blockIdx.y * (R * G); r0 < S.rows; r0 += gridDim.y * (R * G)) {
      float M[R], sum[R];
      f32x4 o[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        M[k] = -INFINITY;
        sum[k] = 0.f;
        o[k] = (f32x4){};
      }
#pragma unroll 2
      for (int i = 0; i < S.parts; ++i) {
        const float* p = A.part + (int64_t)(2 * (w + i) + (i == 0)) * part_floats<DB>(max_rows);
        float mi[R], li[R];
        f32x4 v[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
          const int r = min(r0 + k * G + grp, S.rows - 1);
          mi[k] = p[max_rows * DP + r];
          li[k] = p[max_rows * (DP + 1) + r];
          v[k] = *reinterpret_cast<const f32x4*>(p + (int64_t)r * DP + min(4 * c, DP - 4));
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
          const float top = fmaxf(M[k], mi[k]), t = top == -INFINITY ? 0.f : top;
          const float x = __builtin_amdgcn_exp2f(M[k] - t), y = __builtin_amdgcn_exp2f(mi[k] - t);
          M[k] = top;
          sum[k] = sum[k] * x + li[k] * y;
#pragma unroll
          for (int j = 0; j < 4; ++j) o[k][j] = o[k][j] * x + v[k][j] * y;
        }
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const int r = r0 + k * G + grp, m = S.m0 + r;
        if (r >= S.rows) break;
        const int query = query_of(A, m), head = S.g * A.per + m - query * A.per;
        const int64_t qrow = (int64_t)S.q0 + query;
        const float f = sum[k] == 0.f ? 0.f : 1.f / sum[k];
        typedef T four __attribute__((ext_vector_type(4)));
        if (4 * c < A.d) *reinterpret_cast<four*>((T*)A.o + (qrow * A.heads + head) * A.d + 4 * c) = (four){(T)(o[k][0] * f), (T)(o[k][1] * f), (T)(o[k][2] * f), (T)(o[k][3] * f)};
        if (c == 0 && A.lse) A.lse[(int64_t)head * A.rq + qrow] = sum[k] == 0.f ? -INFINITY : (M[k] + log2f(sum[k])) * kLn2;
      }
    }
    return;
  }
  for (int r0 = blockIdx.y * rows; r0 < S.rows; r0 += gridDim.y * rows) {
    const int r = r0 + grp / split;
    float M = -INFINITY, sum = 0.f;
    f32x4 o = {};
    if (r < S.rows) {
#pragma unroll 4
      for (int i = at; i < S.parts; i += split) {
        // the block's first part is its workgroup's last, the others are their workgroups' first
        const float* p = A.part + (int64_t)(2 * (w + i) + (i == 0)) * part_floats<DB>(max_rows);
        const float mi = p[max_rows * DP + r], li = p[max_rows * (DP + 1) + r];
        const f32x4 v = 4 * c < DP ? *reinterpret_cast<const f32x4*>(p + (int64_t)r * DP + 4 * c) : (f32x4){};
        const float top = fmaxf(M, mi), t = top == -INFINITY ? 0.f : top;
        const float x = __builtin_amdgcn_exp2f(M - t), y = __builtin_amdgcn_exp2f(mi - t);
        M = top;
        sum = sum * x + li * y;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = o[k] * x + v[k] * y;
      }
    }
    if (4 * c < DP)
#pragma unroll
      for (int k = 0; k < 4; ++k) red[grp][4 * c + k] = o[k];
    if (c == 0) {
      red[grp][DP] = M;
      red[grp][DP + 1] = sum;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < rows * DP; e += kThreads) {
      const int q = e / DP, x = e - q * DP, m = S.m0 + r0 + q;
      if (r0 + q >= S.rows) continue;
      float top = -INFINITY;
      for (int i = 0; i < split; ++i) top = fmaxf(top, red[q * split + i][DP]);
      const float t = top == -INFINITY ? 0.f : top;
      float all = 0.f, y = 0.f;
      for (int i = 0; i < split; ++i) {
        const float f = __builtin_amdgcn_exp2f(red[q * split + i][DP] - t);
        all = fmaf(red[q * split + i][DP + 1], f, all);
        y = fmaf(red[q * split + i][x], f, y);
      }
      const int query = query_of(A, m), head = S.g * A.per + m - query * A.per;
      const int64_t qrow = (int64_t)S.q0 + query;
      if (x < A.d) ((T*)A.o)[(qrow * A.heads + head) * A.d + x] = (T)(all == 0.f ? 0.f : y / all);
      if (x == 0 && A.lse) A.lse[(int64_t)head * A.rq + qrow] = all == 0.f ? -INFINITY : (top + log2f(all)) * kLn2;
    }
    __syncthreads();
  }
}

template <typename T, int DB>
hipError_t run_paged(const PArgs& A, int max_rows, hipStream_t st) {
  using M = typename std::conditional<std::is_same<T, float>::value, Split, T>::type;
  constexpr int BYTES = Walk<M, DB>::BYTES;
  hipLaunchKernelGGL((k_paged<M, DB>), dim3(A.W), dim3(kThreads), BYTES, st, A, max_rows);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || A.W == 1) return e;
  hipLaunchKernelGGL((k_paged_join<T, DB>), dim3(A.W - 1, max_rows <= 32 ? 4 : max_rows / 32), dim3(kThreads), 0, st, A, max_rows);
  return hipGetLastError();
}

template <typename T>
hipError_t run_paged_db(const PArgs& A, int max_rows, hipStream_t st) {
  switch ((A.d + 31) / 32) {
    case 1: return run_paged<T, 1>(A, max_rows, st);
    case 2: return run_paged<T, 2>(A, max_rows, st);
    case 3: return run_paged<T, 3>(A, max_rows, st);
    default: return run_paged<T, 4>(A, max_rows, st);
  }
}

inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace
}  // namespace attn
}  // namespace dnb

using namespace dnb::attn;

struct dnb_paged_attn {
  dnb_paged_attn_desc d;
  int W, max_rows, cost[3], extra[3], least;
  size_t ws_part, ws_bytes;
};

extern "C" {

int dnb_paged_attn_create(const dnb_paged_attn_desc* desc, dnb_paged_attn** out) {
  if (!desc || !out) return DNB_E_NULL;
  dnb_paged_attn_desc d = *desc;
  const int rc = dnb::paged::check_layout(desc->cache, &d.cache);
  if (rc != DNB_OK) return rc;
  if (d.heads < 1 || d.heads % d.cache.kv_heads != 0 || d.rows_q < 0 || d.q_stride < 0 || !(d.scale >= 0.f && d.scale < INFINITY)) return DNB_E_BADDESC;
  const int64_t qd = (int64_t)d.heads * d.cache.head_dim, per = d.heads / d.cache.kv_heads, most = 0x7fffffff;
  if (d.q_stride == 0) d.q_stride = qd;
  if (d.scale == 0.f) d.scale = (float)(1.0 / sqrt((double)d.cache.head_dim));
  if (d.heads > 65536 || d.q_stride % (d.cache.dtype == DNB_BF16 ? 8 : 4) != 0 || d.q_stride > (1 << 22) || d.q_stride < qd || d.rows_q > most ||
      d.rows_q * per > most - 256 || d.rows_q * d.heads > most)
    return DNB_E_RANGE;
  dnb_paged_attn* p = new (std::nothrow) dnb_paged_attn();
  if (!p) return DNB_E_NOMEM;
  p->d = d;
  p->W = d.cache.dtype == DNB_F32 && d.cache.head_dim <= 64 ? 512 : 256;
  const int64_t M = d.rows_q * per;
  const bool bf16 = d.cache.dtype == DNB_BF16;
  if (bf16) p->max_rows = M <= 32 ? 32 : M <= 128 ? 128 : 256;
  else p->max_rows = M <= 64 ? 64 : 128;
  // Measured at 16 to 32 heads of 64 and 128, in units of about a thousand cycles: a step, and what a block's beginning and end take (queries,
  // first keys, masked steps, results), for one, two and four sets of rows side by side.  An end that counts too little leaves
  // the workgroups with many short blocks behind: chunks of mixed lengths 690 us with 10 for 40, 505 with 40; 21 single tokens 107 us
  // with 1 for 8, 97 with 2, 72 with 8, 79 with 40.
  const int cost[3] = {5, 5, 8}, extra_bf[3] = {8, 12, 40}, extra_f[3] = {2, 3, 4};
  for (int i = 0; i < 3; ++i) { p->cost[i] = cost[i]; p->extra[i] = bf16 ? extra_bf[i] : extra_f[i]; }
  p->least = 5;  // (one token over 777 keys: 14.8 us, 16.5 with 10, 19 with 20: below that the join's parts cost what is won)
  const int dp = (d.cache.head_dim + 31) / 32 * 32;
  p->ws_part = ((size_t)p->W * sizeof(Shared) + 255) / 256 * 256;
  p->ws_bytes = p->ws_part + (size_t)2 * p->W * p->max_rows * (dp + 2) * sizeof(float);
  *out = p;
  return DNB_OK;
}

void dnb_paged_attn_destroy(dnb_paged_attn* p) { delete p; }

size_t dnb_paged_attn_workspace_bytes(const dnb_paged_attn* p) { return p ? p->ws_bytes : 0; }

int dnb_paged_attn_forward(const dnb_paged_attn* p, const void* q, const void* k_pages, const void* v_pages, const int32_t* q_offsets,
                           const int32_t* k_lengths, const int32_t* table, void* out, float* lse, void* workspace, void* stream) {
  if (!p) return DNB_E_NULL;
  if (p->d.rows_q == 0) return DNB_OK;
  const dnb_paged_layout& c = p->d.cache;
  if (!q || !out || !q_offsets || !k_lengths || !table || !workspace || (c.pages > 0 && (!k_pages || !v_pages))) return DNB_E_NULL;
  for (const void* x : {q, k_pages, v_pages, (const void*)out, (const void*)workspace})
    if (off16(x)) return DNB_E_ALIGN;
  for (const void* x : {(const void*)q_offsets, (const void*)k_lengths, (const void*)table, (const void*)lse})
    if (reinterpret_cast<uintptr_t>(x) & 3u) return DNB_E_ALIGN;
  PArgs A{};
  A.q = q; A.k = k_pages; A.v = v_pages; A.o = out; A.lse = lse;
  A.shared = (Shared*)workspace;
  A.part = (float*)((char*)workspace + p->ws_part);
  A.qo = q_offsets; A.lens = k_lengths; A.table = table;
  A.n = c.sequences; A.heads = p->d.heads; A.kv = c.kv_heads; A.per = p->d.heads / c.kv_heads; A.d = c.head_dim;
  A.causal = p->d.causal != 0; A.columns = c.max_pages; A.shift = dnb::paged::log2_of(c.page_size);
  A.W = p->W;
  for (int i = 0; i < 3; ++i) { A.cost[i] = p->cost[i]; A.extra[i] = p->extra[i]; }
  A.least = p->least;
  A.pages = c.pages; A.rq = p->d.rows_q; A.qs = p->d.q_stride; A.ps = c.page_stride; A.rs = c.row_stride; A.hs = c.head_stride;
  A.c = p->d.scale * kLog2e;
  // m / per = umulhi(m, floor(2^(31 + l) / per) + 1) >> (l - 1) for 2^(l - 1) < per <= 2^l, m below 2^31
  if (A.per > 1) {
    int l = 1;
    while ((1 << l) < A.per) ++l;
    A.per_mul = (uint32_t)(((uint64_t)1 << (31 + l)) / A.per + 1);
    A.per_shift = l - 1;
  }
  const hipError_t e = c.dtype == DNB_BF16 ? run_paged_db<__bf16>(A, p->max_rows, (hipStream_t)stream)
                                           : run_paged_db<float>(A, p->max_rows, (hipStream_t)stream);
  return e == hipSuccess ? DNB_OK : DNB_E_LAUNCH;
}

}  // extern "C"
