// Device helpers of the packed-sequence attention kernels (dnb_attn.hip, dnb_attn_bwd.hip).
//
// One wave works on 32 rows (the columns of its matrix products) against tiles of the other side in
// LDS.  Every product is one of two:
//   row_mul   S[r][c]   = sum_d X[r][d] B[d][c]     X a tile in LDS, B this wave's 32 columns in registers
//   col_mul   Y[d][c]  += sum_r X[r][d] S[r][c]     S as row_mul left it
// With 32x32 products a lane holds column c = lane & 31 of S and its rows 8*(i/4) + 4*(lane>>5) + i%4,
// i < 16.  That is also how the second product wants its right operand, up to an order of the rows over
// which it sums, and any order will do as long as the left operand has the same one: S goes from one
// product into the next without leaving its lane, and a softmax over r is 16 values a lane and one
// exchange between the halves of the wave.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/dnb.h"

namespace dnb {
namespace attn {

// What every kernel of an attention plan is given.  Strides in elements between rows.
struct Args {
  const void *q, *k, *v, *out, *dout;
  void *o, *dq, *dk, *dv;  // o: the forward's output
  float *lse;              // (heads, rows_q)
  float *rowdot;           // backward: sum of dout * out of each row, (heads, rows_q)
  float *part;             // partial results of work that is split

  const int32_t *qo, *ko, *kl;
  int n, heads, kv, per, d, causal;
  int64_t rq, rk, qs, ks, vs, os;
  float scale, c;          // c = scale * log2(e)
  const int64_t *index;    // see Index; null: few sequences
  int waves;               // split work: parts of it, one a wave or a workgroup
  int64_t slots;           //             partial results that `part` has room for
};

namespace {

// A launch has less than 2^32 threads in one dimension, and there may be more tiles, items or rows of heads than
// that takes: workgroups are counted over x, then y.
constexpr unsigned kAcross = 1u << 22;
inline dim3 flat_grid(int64_t count, unsigned z = 1) {
  return count <= (int64_t)kAcross ? dim3((unsigned)count, 1, z) : dim3(kAcross, (unsigned)((count + kAcross - 1) / kAcross), z);
}
__device__ __forceinline__ unsigned flat_block() { return blockIdx.y * kAcross + blockIdx.x; }

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 16 bytes of a row: 8 bf16 or 4 floats
union Piece {
  u32x4 q;
  bf16x8 h;
  __bf16 b[8];
  float f[4];
};

__device__ __forceinline__ int lane_id() { return threadIdx.x & 63; }
// row of element i of a 32x32 result in this lane
__device__ __forceinline__ int row_of(int i) { return 8 * (i >> 2) + 4 * (lane_id() >> 5) + (i & 3); }

__device__ __forceinline__ float half_max(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// fp32 on the matrix cores' bf16 rate: x is the sum of three bf16 (8 bits of its 24 each, every remainder
// exact), and of the nine products of two such sums the six that are not below 2^-23 of the whole are
// made, at 32 cycles each where the fp32 instruction takes 512 for the same: six passes of a sixteenth.  Sums are
// fp32 either way, and so is the error.  Infinities and values above the largest bf16 (3.39e38) have no such sum:
// their remainders are not finite, and every product with them is NaN.  A workgroup whose sums are not finite
// therefore does its work once more with Whole, where the parts' sum is the value, whatever it is, and every
// product is the fp32 instruction's: infinities are then what arithmetic makes of them, at five times the time, and
// hidden ones nothing.
struct Split {};
struct Whole {};
template <typename T>
constexpr bool is_whole = std::is_same<T, Whole>::value;
template <typename T>
constexpr bool in_parts = std::is_same<T, Split>::value || is_whole<T>;
template <typename T>
struct Elem {
  using type = T;
};
template <>
struct Elem<Split> {
  using type = float;
};
template <>
struct Elem<Whole> {
  using type = float;
};
template <typename T>
using elem_t = typename Elem<T>::type;  // of the tensors

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, (bf16x2){(__bf16)a, (__bf16)b});
}
__device__ __forceinline__ void split8(const float (&x)[8], Piece (&p)[3], Split*) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = x[2 * j], b = x[2 * j + 1];
    const unsigned hi = pack_bf16(a, b);
    const float a1 = a - __uint_as_float(hi << 16), b1 = b - __uint_as_float(hi & 0xffff0000u);
    const unsigned mid = pack_bf16(a1, b1);
    p[0].q[j] = hi;
    p[1].q[j] = mid;
    p[2].q[j] = pack_bf16(a1 - __uint_as_float(mid << 16), b1 - __uint_as_float(mid & 0xffff0000u));
  }
}
__device__ __forceinline__ void split8(const float (&x)[8], Piece (&p)[3], Whole*) {
  constexpr float kMost = 3.3895313892515355e38f;  // the largest bf16
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool inf = fabsf(x[j]) == INFINITY;
    const float hi = inf || !(fabsf(x[j]) > kMost) ? (float)(__bf16)x[j] : copysignf(kMost, x[j]);
    const float rest = inf ? 0.f : x[j] - hi;
    const float mid = (float)(__bf16)rest;
    p[0].b[j] = (__bf16)hi;
    p[1].b[j] = (__bf16)mid;
    p[2].b[j] = (__bf16)(rest - mid);
  }
}
// ... of 8 floats as loaded
template <typename T>
__device__ __forceinline__ void split8(const u32x4& lo, const u32x4& hi, Piece (&p)[3]) {
  float x[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = __uint_as_float(lo[j]);
    x[4 + j] = __uint_as_float(hi[j]);
  }
  split8(x, p, (T*)nullptr);
}

// A tile in LDS: rows of PC pieces of 16 bytes, of which CH hold the row (head_dim padded with zeros to
// DB blocks of 32).  Piece c of row r lies at c ^ swz(r): sixteen rows read at one c (row_mul), and four
// rows read 64 bytes wide (col_mul in bf16) or rows r and r + 4 read 128 bytes wide (in fp32), each meet
// all the banks.  Each bit of swz is one of r's, so swz(r + s) is swz(r) ^ swz(s) where r and s share no bit.
// In parts: PL tiles, of the first, second and third.
template <typename T, int DB>
struct Tile {
  static constexpr bool BF = !std::is_same<T, float>::value;
  static constexpr int PL = in_parts<T> ? 3 : 1;
  static constexpr int EP = BF ? 8 : 4;                // elements of a piece
  static constexpr int LD = EP * sizeof(elem_t<T>) / 16;  // loads of a piece from memory
  static constexpr int CH = DB * 32 / EP;
  static constexpr int PC = BF ? (DB == 1 ? 4 : DB == 2 ? 8 : 16) : (DB == 1 ? 8 : DB == 2 ? 16 : 32);
  static constexpr int PITCH = PC * 16;                // bytes
  static constexpr int NS = CH / 2;                    // steps of row_mul: a lane's half of the wave takes piece 2s + half
  static constexpr int ROWS = std::is_same<T, __bf16>::value ? 64 : 32;  // rows of a shared tile
  static constexpr int BYTES = ROWS * PITCH * PL;
  static __device__ __forceinline__ constexpr int swz(int r) {
    if constexpr (BF) {
      if constexpr (PC == 4) return (r >> 2) & 3;
      else if constexpr (PC == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
      else return ((r & 3) << 2) | ((r >> 2) & 3);
    } else {
      if constexpr (PC == 8) return (r >> 1) & 7;
      else return (((r >> 2) & 1) << 3) | (((r >> 3) & 1) << 2) | (r & 3);
    }
  }
  static __device__ __forceinline__ int at(int r, int c) { return r * PITCH + ((c ^ swz(r)) << 4); }
};

// Whether the waves of a workgroup of k_attn and k_attn_dq share the keys out in halves.  Eight waves at one
// barrier are slower than two workgroups of four (12597 packed queries of 32 heads: 471 us for 393), but
// with fewer tiles than compute units a workgroup's time is the launch's (1500 rows of 4 heads, a step: 152 us
// for 170), unless the keys are one step anyway (a step of 33 tokens: 27 us for 24).  Four / eight waves, us of the
// forward of 8 heads of 128: bf16 128 keys 6.7 / 7.6, 256 8.8 / 9.3, 512 13.0 / 12.7, 1024 21.6 / 19.6, 4096 71.7 / 60.5; fp32
// 128 17.5 / 16.7, 256 27.8 / 25.6, 1024 93.3 / 75.8; at 384 tiles of 2048 keys still 48.9 / 46.1 and 197.8 / 194.1.
inline bool split_keys(const Args& A, int64_t tiles) { return tiles * A.kv <= 256 && A.rk >= 256 * (int64_t)A.n; }

// Copies of a step's tiles in LDS: the next one is written while one is read, unless the tiles are so large
// that a second workgroup on the compute unit does more (in parts above head_dim 64: 48 KB a copy).
template <typename T>
constexpr int buffers(int blocks) { return in_parts<T> && blocks > 2 ? 1 : 2; }

// 16 bytes of a tile, or of each of its three
template <typename T, int DB>
using Pieces = Piece[Tile<T, DB>::PL];
// a wave's 32 columns: of each step, this lane's half
template <typename T, int DB>
struct ColumnsOf {
  using type = Pieces<T, DB>[Tile<T, DB>::NS];
};
// Whole: where they are in memory, read at every use.  What is done so seldom must not take registers from Split.
struct Row {
  const float* at;
  int d;  // 0: zeros
};
template <int DB>
struct ColumnsOf<Whole, DB> {
  using type = Row;
};
template <typename T, int DB>
using Columns = typename ColumnsOf<T, DB>::type;

__device__ __forceinline__ void mma(f32x16& acc, const Piece (&a)[1], const Piece (&b)[1], __bf16*) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0].h, b[0].h, acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16& acc, const Piece (&a)[1], const Piece (&b)[1], float*) {
#pragma unroll
  for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[0].f[j], b[0].f[j], acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16& acc, const Piece (&a)[3], const Piece (&b)[3], Split*) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0].h, b[2].h, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[2].h, b[0].h, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1].h, b[1].h, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0].h, b[1].h, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1].h, b[0].h, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0].h, b[0].h, acc, 0, 0, 0);
}
// (a lane's eight of the 16 steps of the bf16 instruction are eight instructions of two steps, one of each half.
// Second and third part first: the first two of the largest values add up to 2^128.)
__device__ __forceinline__ float whole(const Piece (&p)[3], int j) { return (float)p[0].b[j] + ((float)p[1].b[j] + (float)p[2].b[j]); }
__device__ __forceinline__ void mma(f32x16& acc, const Piece (&a)[3], const Piece (&b)[3], Whole*) {
#pragma unroll
  for (int j = 0; j < 8; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(whole(a, j), whole(b, j), acc, 0, 0, 0);
}

// Addresses in LDS as bytes from its start: what differs between a wave's reads of a tile is then a
// constant that the instruction holds, or one that is xored to a common address.
typedef uint32_t lds_t;
template <typename V>
__device__ __forceinline__ V lds_read(lds_t at) {
  return *(const __attribute__((address_space(3))) V*)(uintptr_t)at;
}
template <typename V>
__device__ __forceinline__ void lds_write(lds_t at, const V& v) {
  *(__attribute__((address_space(3))) V*)(uintptr_t)at = v;
}
// The kernels have no LDS but what the launch gives them, which starts at 0: a constant, so that it goes into
// the instructions (31 additions a step of k_attn less than with the address of the array).
__device__ __forceinline__ constexpr lds_t lds_start(const void*) { return 0; }
// Keeps the compiler from holding every address derived from `a` in a register of its own over a whole
// loop: with dk, dv and a step's tiles in registers there is no room for them, and a spilled address is
// read back behind the loads of the next tile, for which it then waits.
// (HOLD: where there is room it may do so, which saves an instruction a read: k_attn, 211 -> 247
// registers, 452 -> 383 us for 12597 packed queries of 32 heads.)
template <bool HOLD = false>
__device__ __forceinline__ lds_t at_hand(lds_t a) {
  if (!HOLD) asm volatile("" : "+v"(a));
  return a;
}
// piece `half` of row row0 + (lane & 31) of a tile; piece 2k + half is at this ^ (k << 5)
template <typename T, int DB, bool HOLD = false>
__device__ __forceinline__ lds_t row_address(int row0) {
  return at_hand<HOLD>(Tile<T, DB>::at(row0 + (lane_id() & 31), lane_id() >> 5));
}

// rows row0 .. row0 + 31 of the tile times this wave's columns; TR: rows of the whole tile
template <typename T, int DB, bool HOLD = false, int TR = 32>
__device__ __forceinline__ f32x16 row_mul(lds_t tile, int row0, const Columns<T, DB>& b) {
  using L = Tile<T, DB>;
  const lds_t at = row_address<T, DB, HOLD>(row0);
  f32x16 s = {};
  auto piece = [&](int k, Pieces<T, DB>& a) {
#pragma unroll
    for (int p = 0; p < L::PL; ++p) a[p].q = lds_read<u32x4>((at ^ (k << 5)) + (tile + p * TR * L::PITCH));
  };
  if constexpr (is_whole<T>) {
#pragma unroll 1
    for (int k = 0; k < L::NS; ++k) {
      Pieces<T, DB> a;
      piece(k, a);
      const int e = (2 * k + (lane_id() >> 5)) * L::EP;
#pragma unroll
      for (int j = 0; j < L::EP; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(whole(a, j), e < b.d ? b.at[e + j] : 0.f, s, 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int k = 0; k < L::NS; ++k) {
      Pieces<T, DB> a;
      piece(k, a);
      mma(s, a, b[k], (T*)nullptr);
    }
  }
  return s;
}

// acc += X^T S over eight rows a lane, S from element s0 on, where a weight of 0 takes nothing of a value, whatever that is:
// hidden pairs have that weight.  What is not finite is left out of the product and counted: infinities that
// arrive with either sign, and NaN.
__device__ __forceinline__ void whole_mul(f32x16& acc, const Piece (&x)[3], const f32x16& s, int s0) {
  float v[8], odd = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = whole(x, j);
    const bool fin = fabsf(v[j]) < INFINITY;
    odd = fin ? odd : 1.f;
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(fin ? v[j] : 0.f, s[s0 + j], acc, 0, 0, 0);
  }
  if (!__any(odd != 0.f)) return;
  auto one = [](bool b) { return b ? 1.f : 0.f; };
#pragma unroll
  for (int kind = 0; kind < 3; ++kind) {
    const float to = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
    f32x16 count = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float w = s[s0 + j];
      if (kind == 2) {
        count = __builtin_amdgcn_mfma_f32_32x32x2f32(one(v[j] != v[j]), one(w < 0.f || w > 0.f), count, 0, 0, 0);
      } else {
        count = __builtin_amdgcn_mfma_f32_32x32x2f32(one(v[j] == to), one(w > 0.f), count, 0, 0, 0);
        count = __builtin_amdgcn_mfma_f32_32x32x2f32(one(v[j] == -to), one(w < 0.f), count, 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] += count[i] > 0.f ? to : 0.f;
  }
}

// bf16: rounding s to 8 bits of mantissa is what feeding the matrix cores at their bf16 rate costs;
// the sums stay in fp32.
template <typename T, int DB, bool HOLD = false, int TR = 32>
__device__ __forceinline__ void col_mul(lds_t tile, int row0, const f32x16& s, f32x16 (&acc)[DB]) {
  using L = Tile<T, DB>;
  const int l = lane_id();
  if constexpr (L::BF) {
    // row0 is a multiple of 32: rows 8 on lie at piece ^ 2, rows 16 on at the same pieces
    const lds_t at = at_hand<HOLD>(L::at(row0 + 4 * (l >> 5) + ((l >> 2) & 3), 2 * ((l >> 4) & 1) + ((l >> 1) & 1)) + (l & 1) * 8);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      Pieces<T, DB> y;
      if constexpr (is_whole<T>) {
      } else if constexpr (L::PL == 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[0].b[j] = (__bf16)s[8 * t + j];
      } else {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = s[8 * t + j];
        split8(v, y, (T*)nullptr);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        Pieces<T, DB> x;
#pragma unroll
        for (int p = 0; p < L::PL; ++p) {
          using lds4 = __attribute__((address_space(3))) s16x4;
          const lds_t from = tile + p * TR * L::PITCH + 16 * t * L::PITCH;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(uintptr_t)((at ^ (db << 6)) + from));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(uintptr_t)((at ^ (db << 6) ^ 32) + (from + 8 * L::PITCH)));
          const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
          x[p].q = (u32x4){a.x, a.y, b.x, b.y};
        }
        if constexpr (is_whole<T>) {
          whole_mul(acc[db], x, s, 8 * t);
          __builtin_amdgcn_sched_barrier(0);  // no reads ahead, no registers for them
        } else {
          mma(acc[db], x, y, (T*)nullptr);
        }
      }
    }
  } else {
    const lds_t at = at_hand<HOLD>(L::at(row0 + 4 * (l >> 5), (l & 31) >> 2) + (l & 3) * 4);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = 8 * (i >> 2) + (i & 3);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const float x = lds_read<float>((at ^ (db << 7) ^ (L::swz(r) << 4)) + (tile + r * L::PITCH));
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[i], acc[db], 0, 0, 0);
      }
    }
  }
}

// An order for the compiler's scheduler: N products, each with a read of LDS, AHEAD reads before the first.
template <int AHEAD, int N>
__device__ __forceinline__ void read_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// A loaded piece to its place in a tile of TR rows
template <typename T, int DB, int TR>
__device__ __forceinline__ void write_piece(lds_t to, const u32x4* r) {
  using L = Tile<T, DB>;
  if constexpr (L::PL == 1) {
    lds_write(to, r[0]);
  } else {
    Piece p[3];
    split8<T>(r[0], r[1], p);
#pragma unroll
    for (int i = 0; i < 3; ++i) lds_write(to + i * TR * L::PITCH, p[i].q);
  }
}
// Pieces tid, tid + NT, ... of a tile's TR rows
template <typename T, int DB, int U, int NT, int TR>
__device__ __forceinline__ void store_pieces(lds_t tile, int tid, const u32x4 (&r)[U * Tile<T, DB>::LD]) {
  using L = Tile<T, DB>;
  if constexpr (NT % L::CH == 0) {
    constexpr int STEP = NT / L::CH;  // a power of two, above the thread's first row
    const lds_t at = at_hand(L::at(tid / L::CH, tid % L::CH));
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (TR * L::CH % NT == 0 || tid + u * NT < TR * L::CH)
        write_piece<T, DB, TR>((at ^ (L::swz(u * STEP) << 4)) + (tile + u * STEP * L::PITCH), r + u * L::LD);
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = tid + u * NT, row = i / L::CH, c = i - row * L::CH;
      if (TR * L::CH % NT == 0 || i < TR * L::CH) write_piece<T, DB, TR>(tile + L::at(row, c), r + u * L::LD);
    }
  }
}

// Rows of a tile on their way from memory to LDS, NT threads.  The loads go through a buffer descriptor
// over exactly the rows that exist: what lies past them, and the pieces that pad head_dim, reads as zero.
template <typename T, int DB, int ROWS, int NT>
struct Stage {
  using L = Tile<T, DB>;
  using E = elem_t<T>;
  static constexpr int U = (ROWS * L::CH + NT - 1) / NT;
  u32x4 r[U * L::LD];
  uint32_t off[U];
  __device__ __forceinline__ void init(int tid, int64_t stride, int d) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = tid + u * NT, row = i / L::CH, c = i - row * L::CH;
      off[u] = c * L::EP < d && row < ROWS ? (uint32_t)(row * (int)stride + c * L::EP) * (uint32_t)sizeof(E) : 0x80000000u;
    }
  }
  // base: the first row; rows: how many there are from it on (uniform in the wave; 0 or less: none)
  __device__ __forceinline__ void load(const E* base, int64_t stride, int rows, int d) {
    const int n = rows > ROWS ? ROWS : rows;
    const int bytes = n > 0 ? (int)(((n - 1) * (int)stride + d) * (int)sizeof(E)) : 0;
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00027000);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int p = 0; p < L::LD; ++p) r[u * L::LD + p] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off[u] + 16 * p, 0, 0);
  }
  __device__ __forceinline__ void store(lds_t tile, int tid) { store_pieces<T, DB, U, NT, ROWS>(tile, tid, r); }
};

// This lane's column (its half of each step's two pieces) of a row of d elements; zeros if !valid.
template <typename T, int DB>
__device__ __forceinline__ void load_cols(Columns<T, DB>& f, const elem_t<T>* row, bool valid, int d) {
  using L = Tile<T, DB>;
  if constexpr (is_whole<T>) {
    f = {row, valid ? d : 0};
  } else {
    const int h = lane_id() >> 5;
#pragma unroll
    for (int k = 0; k < L::NS; ++k) {
      const int e = (2 * k + h) * L::EP;
      u32x4 x[L::LD];
#pragma unroll
      for (int p = 0; p < L::LD; ++p) {
        x[p] = (u32x4){0u, 0u, 0u, 0u};
        if (valid && e < d) x[p] = *reinterpret_cast<const u32x4*>(row + e + p * (L::EP / L::LD));
      }
      if constexpr (L::PL == 1) f[k][0].q = x[0];
      else split8<T>(x[0], x[1], f[k]);
    }
  }
}
// The product of two rows of d elements, half of it in each half of the wave
template <typename T, int DB>
__device__ __forceinline__ float dot_rows(const elem_t<T>* a, const elem_t<T>* b, bool valid, int d) {
  constexpr int EP = 16 / sizeof(elem_t<T>);
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < 32 * DB / EP; k += 2) {
    const int e = (k + (lane_id() >> 5)) * EP;
    Piece x, y;
    x.q = y.q = (u32x4){0u, 0u, 0u, 0u};
    if (valid && e < d) {
      x.q = *reinterpret_cast<const u32x4*>(a + e);
      y.q = *reinterpret_cast<const u32x4*>(b + e);
    }
#pragma unroll
    for (int j = 0; j < EP; ++j) {
      if constexpr (sizeof(elem_t<T>) == 2) s = fmaf((float)x.b[j], (float)y.b[j], s);
      else s = fmaf(x.f[j], y.f[j], s);
    }
  }
  return half_sum(s);
}

// Y[d][c] of a wave (col_mul's result) times f into row c
template <typename T, int DB>
__device__ __forceinline__ void store_cols(T* row, bool valid, int d, const f32x16 (&acc)[DB], float f) {
  if (!valid) return;
  const int h = lane_id() >> 5;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int e = 32 * db + 8 * g + 4 * h;
      if (e >= d) continue;
      if constexpr (sizeof(T) == 2) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = (__bf16)(acc[db][4 * g + j] * f);
        *reinterpret_cast<bf16x4*>(row + e) = y;
      } else {
        *reinterpret_cast<float4*>(row + e) =
            make_float4(acc[db][4 * g] * f, acc[db][4 * g + 1] * f, acc[db][4 * g + 2] * f, acc[db][4 * g + 3] * f);
      }
    }
}

// Whether some value of the wave's is infinite or NaN
template <int DB>
__device__ __forceinline__ bool not_finite(const f32x16 (&acc)[DB]) {
  float t = 0.f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) t = fmaf(acc[db][i], 0.f, t);
  return __any(t != t);
}
// x in a form in which Whole's walk does not share it, or what is made of it, with the walk before: it would take a
// register through all of that.
template <typename F, typename X>
__device__ __forceinline__ X apart(X x) {
  if (is_whole<F>) asm volatile("" : "+v"(x));
  return x;
}
// v of any of the workgroup's WAVES waves, through kFlags bytes of LDS at `at`
constexpr int kFlags = 64;
template <int WAVES>
__device__ __forceinline__ bool any_wave(lds_t at, bool v) {
  if (lane_id() == 0) lds_write(at + 4 * (threadIdx.x >> 6), (int)v);
  __syncthreads();
  int any = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) any |= lds_read<int>(at + 4 * w);
  return __builtin_amdgcn_readfirstlane(any) != 0;
}

// One sequence, as its offsets say; whatever they hold, the rows stay inside the tensors.  nk may be 2^31 - 1:
// positions of keys, which go up to a tile further, are unsigned.
struct Seq {
  int q0, nq, k0, nk, span;  // span: rows of k up to the next sequence's, of which nk are in use
};
__device__ __forceinline__ Seq seq_at(const Args& A, int i) {
  Seq s;
  const int64_t q0 = min(max((int64_t)A.qo[i], (int64_t)0), A.rq), q1 = min(max((int64_t)A.qo[i + 1], q0), A.rq);
  const int64_t k0 = min(max((int64_t)A.ko[i], (int64_t)0), A.rk), k1 = min(max((int64_t)A.ko[i + 1], k0), A.rk);
  s.q0 = (int)q0; s.nq = (int)(q1 - q0); s.k0 = (int)k0; s.span = (int)(k1 - k0);
  s.nk = A.kl ? min(max(A.kl[i], 0), s.span) : s.span;
  return s;
}

// v of the lane that CTRL names, 0 where there is none or ROWS (of 16 lanes, a bit each) leaves this one out
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t from_lane(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
// Inclusive sum over the lanes, within the registers: through LDS it took 0.7 us of every kernel here.
__device__ __forceinline__ int64_t wave_scan(int64_t v) {
  v += from_lane<0x111, 0xf>(v);  // 1, 2, 4 and 8 lanes down inside a row
  v += from_lane<0x112, 0xf>(v);
  v += from_lane<0x114, 0xf>(v);
  v += from_lane<0x118, 0xf>(v);
  v += from_lane<0x142, 0xa>(v);  // lane 15 to row 1, lane 47 to row 3
  v += from_lane<0x143, 0xc>(v);  // lane 31 to rows 2 and 3
  return v;
}
__device__ __forceinline__ int bcast(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ Seq bcast(const Seq& s, int lane) {
  return {bcast(s.q0, lane), bcast(s.nq, lane), bcast(s.k0, lane), bcast(s.nk, lane), bcast(s.span, lane)};
}
__device__ __forceinline__ int64_t bcast64(int64_t v, int lane) {
  return (int64_t)(((uint64_t)(uint32_t)bcast((int)(v >> 32), lane) << 32) | (uint32_t)bcast((int)v, lane));
}

// Index of many sequences, made by k_attn_index before the kernels that search: sums over the sequences before
// chunk c of 64, for c = 0 .. chunks, of the numbers below.  Every wave finds its work in the offsets by itself, 64
// sequences at a time; without the index that is a walk through all chunks for every tile, part and row, and
// their product is what 4096 requests of one token over 256 keys (32 heads) took 7.1 ms for, 0.77 with the index,
// and 40.9 ms for their gradients, 4.0 with it.
// Up to so many sequences the walk is no longer than the launch.  Measured without and with the index, us: split, one
// token over 256 keys each, forward 31 / 33 (128 sequences), 47 / 43 (192), gradients 105 / 106, 209 / 184; tiles, 33
// tokens of 8 heads each, forward 18 / 21 (256), 24 / 26 (384), 35 / 31 (512), gradients 47 / 50 (128), 59 / 59 (192),
// 57 / 53 (256).
enum { kTiles, kUnits, kItems, kCost, kKeyItems, kSums };
constexpr int kScanSplit = 128, kScanBackward = 192, kScanForward = 384;
__host__ __device__ inline int chunks_of(int n) { return (n + 63) / 64; }
inline size_t index_bytes(int n) { return n > kScanSplit ? (size_t)kSums * (chunks_of(n) + 1) * sizeof(int64_t) : 0; }
__device__ __forceinline__ const int64_t* index_of(const Args& A, int kind) { return A.index + kind * (chunks_of(A.n) + 1); }
// of sums p[0] .. p[count], the c with p[c] <= x < p[c + 1]; count if x is not below p[count]
__device__ __forceinline__ int index_find(const int64_t* p, int count, int64_t x) {
  int lo = 0, len = count;
  for (;;) {
    const int step = (len + 63) / 64, end = min((lane_id() + 1) * step, len);
    const uint64_t past = __ballot(p[lo + end] > x);
    if (!past) return count;
    const int at = __builtin_ctzll(past);
    lo += at * step;
    len = min(step, len - at * step);
    if (step == 1) return lo;
  }
}
// F::sums(A, sequence, v) sets the first F::N numbers.  One workgroup.
constexpr int kIndexThreads = 1024;
template <typename F>
__global__ __launch_bounds__(kIndexThreads) void k_attn_index(Args A, int64_t* to) {
  const int l = lane_id(), wave = threadIdx.x >> 6, count = chunks_of(A.n);
  for (int c = wave; c < count; c += kIndexThreads / 64) {
    int64_t v[F::N] = {};
    if (c * 64 + l < A.n) F::sums(A, seq_at(A, c * 64 + l), v);
#pragma unroll
    for (int k = 0; k < F::N; ++k) {
      const int64_t sum = wave_scan(v[k]);
      if (l == 63) to[k * (count + 1) + c + 1] = sum;
    }
  }
  __syncthreads();
  if (wave >= F::N) return;
  int64_t* p = to + wave * (count + 1);
  int64_t before = 0;
  if (l == 0) p[0] = 0;
  for (int c = 0; c < count; c += 64) {
    const int64_t sum = before + wave_scan(c + l < count ? p[c + l + 1] : 0);
    if (c + l < count) p[c + l + 1] = sum;
    before = bcast64(sum, 63);
  }
}

// The sequence that tile number `tile` of all sequences' tiles of 128 rows belongs to, and its number there.
// No host copy comes before.  False: there are fewer tiles.
constexpr int kRows = 128;  // packed rows of a workgroup of k_attn and k_attn_dq, 32 a wave
__device__ __forceinline__ int tiles_of(const Args& A, const Seq& s) { return (int)(((int64_t)s.nq * A.per + kRows - 1) / kRows); }
__device__ __forceinline__ bool find_tile(const Args& A, int64_t tile, Seq* s, int* t, int* count) {
  const int l = lane_id();
  int64_t base = 0;
  int i0 = 0;
  if (A.index) {
    const int64_t* p = index_of(A, kTiles);
    const int c = index_find(p, chunks_of(A.n), tile);
    if (c == chunks_of(A.n)) return false;
    i0 = c * 64;
    base = p[c];
  }
  for (; i0 < A.n; i0 += 64) {
    Seq mine = {};
    int c = 0;
    if (i0 + l < A.n) {
      mine = seq_at(A, i0 + l);
      c = tiles_of(A, mine);
    }
    const int64_t end = wave_scan(c);
    const uint64_t past = __ballot(base + end > tile);
    if (past) {
      const int at = __builtin_ctzll(past);
      *s = bcast(mine, at);
      *count = bcast(c, at);
      *t = (int)(tile - base - (bcast64(end, at) - *count));
      return true;
    }
    base += bcast64(end, 63);
  }
  return false;
}

// 32 packed rows of a wave, a lane's own being m0 + (lane & 31)
struct RowTile {
  bool valid;
  int head;
  unsigned sees, most, least;  // keys that the lane's row sees; that the wave's last row, its first row see
  int64_t qrow;
  static __device__ __forceinline__ unsigned seen(const Args& A, const Seq& S, int m) {
    return A.causal ? max(S.nk + min(m / A.per + 1 - S.nq, 0), 0) : S.nk;
  }
  __device__ __forceinline__ RowTile(const Args& A, const Seq& S, int g, int m0) {
    const int M = S.nq * A.per, m = m0 + (lane_id() & 31), row = m / A.per;
    valid = m < M;
    head = g * A.per + m - row * A.per;
    qrow = (int64_t)S.q0 + row;
    sees = seen(A, S, m);
    most = m0 >= M ? 0 : seen(A, S, min(m0 + 31, M - 1));
    least = seen(A, S, m0);
  }
};

// ---- work split over the keys.  Items are (sequence, tile of 32 packed rows, key/value head), in that order,
// a unit is 32 keys of an item, and all units of all items lie on one line, which is cut into equal parts,
// one a wave: whatever the lengths, no wave has more than one unit more than another.  A part of an item
// leaves its result in slot (wave + item): walking along the line, each next part has a next wave or a next
// item.
constexpr int kItemRows = 32, kUnit = 32;
__device__ __forceinline__ int units_of(unsigned keys) { return (int)((keys + kUnit - 1) / kUnit); }

// The rule: where tiles of 128 rows are so few that most of the chip would be idle, or mostly empty, and the
// keys are long enough to be worth the second launch.  Lengths are on the device; the longest sequence is
// taken to have about twice the average's keys.
// Measured at head_dim 128, us of the forward split / in tiles (one sequence, causal, heads = tiles of a row of tiles):
//   bf16  1 query of 8 heads   512 keys 13.4 / 12.7   1024 14.5 / 19.6   4096 16.6 / 60.5
//         128 of 16 (32 tiles) 512 keys 23.8 / 15.9   1024 28.5 / 23.5   4096 33.2 / 69.9;  384 of 16 (64) 4096 56.5 / 71.2
//   fp32  1 query of 8 heads   128 keys 18.3 / 16.7    256 18.3 / 25.6   1024 19.2 / 75.8
//         128 of 32 (64 tiles) 256 keys 33.9 / 29.5    512 39.5 / 47.8   1024 52.9 / 86.0;  64 of 8 of 4 sequences (96)
//         512 63.5 / 49.0, 2048 150.9 / 162.2
// So it is right where it matters most, within a third around 512 keys in bf16, and wrong by 2 to 3 times (some 15 us) for
// several sequences of equal length whose few rows make more tiles than it thinks of: 16 of 8 queries of 32/8
// heads over 256 keys each, bf16, 26.1 / 9.3.  Unequal ones are what it is for.
inline bool split_rows(int64_t rq, int64_t rk, int64_t n, int64_t kv, int64_t per, bool bf16) {
  const int64_t tiles = (rq * per / 128 + n) * kv;
  return (rq * per <= kItemRows * n || tiles <= (bf16 ? 40 : 96)) && 2 * rk >= (n + 1) * (bf16 ? 400 : 256);
}

struct Line {
  int64_t units, items;  // of this lane's sequence
};
__device__ __forceinline__ Line line_of(const Args& A, const Seq& s) {
  const int64_t items = ((int64_t)s.nq * A.per + kItemRows - 1) / kItemRows * A.kv;
  return {items * units_of(s.nk), items};
}
struct RowSums {
  static constexpr int N = 3;
  static __device__ __forceinline__ void sums(const Args& A, const Seq& s, int64_t* v) {
    const Line ln = line_of(A, s);
    v[kTiles] = tiles_of(A, s);
    v[kUnits] = ln.units;
    v[kItems] = ln.items;
  }
};
__device__ __forceinline__ int64_t line_total(const Args& A) {
  if (A.index) return index_of(A, kUnits)[chunks_of(A.n)];
  int64_t u = 0;
  for (int i = lane_id(); i < A.n; i += 64) u += line_of(A, seq_at(A, i)).units;
  return bcast64(wave_scan(u), 63);
}
constexpr int64_t slot_floats(int dp) { return (int64_t)kItemRows * dp + 2 * kItemRows; }

// f(sequence, key/value head, first packed row, first unit, unit after the last, slot) for every part of wave w.
// Where on the line it is is looked up again for every part: what the search needs would not fit the registers
// beside what f keeps.
template <typename F>
__device__ __forceinline__ void each_part(const Args& A, int64_t w, F f) {
  const int l = lane_id();
  const int64_t total = line_total(A), W = min((int64_t)A.waves, total);
  if (w >= W) return;
  int64_t a = w * total / W;
  const int64_t b = (w + 1) * total / W;
  while (a < b) {
    int64_t u0 = 0, i0 = 0, j = 0, slot = -1;  // units and items before the 64 sequences at hand
    Seq S = {};
    int first = 0, last = 0, base = 0;
    if (A.index) {
      const int c = index_find(index_of(A, kUnits), chunks_of(A.n), a);
      base = c * 64;
      u0 = index_of(A, kUnits)[c];
      i0 = index_of(A, kItems)[c];
    }
    for (; base < A.n; base += 64) {
      Seq mine = {};
      Line ln = {};
      if (base + l < A.n) {
        mine = seq_at(A, base + l);
        ln = line_of(A, mine);
      }
      const int64_t ue = wave_scan(ln.units), ie = wave_scan(ln.items);
      const uint64_t past = __ballot(u0 + ue > a);
      if (past) {
        const int at = __builtin_ctzll(past);
        S = bcast(mine, at);
        const int64_t in = a - u0 - bcast64(ue - ln.units, at);
        const int len = units_of(S.nk);
        j = in / len;
        first = (int)(in - j * len);
        last = (int)min((int64_t)len, first + b - a);
        slot = w + i0 + bcast64(ie - ln.items, at) + j;
        break;
      }
      u0 += bcast64(ue, 63);
      i0 += bcast64(ie, 63);
    }
    if (slot < 0 || slot >= A.slots) return;  // offsets that decrease
    f(S, (int)(j % A.kv), (int)(j / A.kv) * kItemRows, first, last, slot);
    a += last - first;
  }
}

// The parts of row id of (query rows, heads): n of them from `slot` on, in each of which it is row r.
struct RowParts {
  bool found;
  int head, r, n;
  int64_t qrow, slot;
};
__device__ __forceinline__ RowParts row_parts(const Args& A, int64_t id) {
  const int l = lane_id();
  RowParts P = {};
  P.qrow = id / A.heads;
  P.head = (int)(id - P.qrow * A.heads);
  int64_t u0 = 0, i0 = 0, su = 0, si = 0;
  Seq S = {};
  int base = 0, end = A.n;
  if (A.index) {
    // the last chunk whose first row is not past this one
    int lo = 0;
    for (int len = chunks_of(A.n); len > 1;) {
      const int step = (len + 63) / 64;
      const int ok = (int)__popcll(__ballot(l * step < len && A.qo[(lo + l * step) * 64] <= P.qrow));
      const int at = ok > 0 ? ok - 1 : 0;  // (none: a row before the first sequence's)
      lo += at * step;
      len = min(step, len - at * step);
    }
    base = lo * 64;
    end = min(base + 64, A.n);
    u0 = index_of(A, kUnits)[lo];
    i0 = index_of(A, kItems)[lo];
  }
  for (; base < end; base += 64) {
    Seq mine = {};
    Line ln = {};
    if (base + l < A.n) {
      mine = seq_at(A, base + l);
      ln = line_of(A, mine);
    }
    const int64_t ue = wave_scan(ln.units), ie = wave_scan(ln.items);
    const uint64_t holds = __ballot(mine.q0 <= P.qrow && P.qrow < (int64_t)mine.q0 + mine.nq);
    if (holds) {
      const int at = __builtin_ctzll(holds);
      S = bcast(mine, at);
      su = u0 + bcast64(ue - ln.units, at);
      si = i0 + bcast64(ie - ln.items, at);
      P.found = true;
    }
    u0 += bcast64(ue, 63);
    i0 += bcast64(ie, 63);
  }
  const int len = units_of(S.nk);
  if (!P.found || len == 0) return P;
  const int64_t total = A.index ? line_total(A) : u0, W = min((int64_t)A.waves, total);
  const int g = P.head / A.per, m = (int)(P.qrow - S.q0) * A.per + P.head - g * A.per;
  const int64_t j = (int64_t)(m / kItemRows) * A.kv + g, first = su + j * len;
  // unit u is wave ((u + 1) W - 1) / total's
  const int64_t w0 = ((first + 1) * W - 1) / total, w1 = ((first + len) * W - 1) / total;
  P.r = m % kItemRows;
  P.n = (int)(w1 - w0 + 1);
  P.slot = si + j + w0;
  if (P.slot + P.n > A.slots) P.found = false;  // offsets that decrease
  return P;
}

}  // namespace
}  // namespace attn
}  // namespace dnb
