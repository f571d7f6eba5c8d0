// The gated delta rule inside packed documents on the matrix cores, forward and backward, of one element type (bf16, half and float each build it:
// delta_rule_*.hip).
//
// With a = exp(g), a token's state is S_t = a_t S_(t-1) + k_t u_t^T, u_t = beta_t (v_t - a_t S_(t-1)^T k_t), and its result scale S_t^T q_t.  A document is
// cut into chunks of 64 tokens.  With G the running sum of a chunk's g, D_ij = exp(G_i - G_j) for j <= i, and S the state before the chunk, the u of
// its tokens solve (1 + A) U = beta (V - exp(G) K S), A_ij = beta_i D_ij k_i.k_j for j < i, so that with T = (1 + A)^-1
//   U = T beta (V - exp(G) K S),  O = scale (exp(G) Q S + P U), P = D o Q K^T,  S' = exp(G_last) S + K^T (exp(G_last - G) U).
// Backward, from dO and dS' (o: element by element):
//   dU = scale P^T dO + exp(G_last - G) K dS',  Y = T^T dU,  dV = beta Y,
//   dS = exp(G_last) dS' + scale Q^T (exp(G) dO) - K^T (beta exp(G) Y),
//   dQ = scale (exp(G) dO S^T + M K),  M = D o dO U^T,  H = -beta D o Y U^T (below the diagonal),
//   dK = -beta exp(G) Y S^T + exp(G_last - G) U dS'^T + scale M^T Q + (H + H^T) K,
// and dbeta and dg from the same products' sums over rows and columns; dg is the sum of dG from a token to its chunk's end.
//
// Three steps: what a chunk has of its own (delta_prep_kernel: T and P, all chunks side by side), the walk from chunk to chunk (delta_walk: the state
// and, backward, its gradient, which needs nothing of the forward walk, so that both share a launch), and the gradients of all chunks side by side
// (delta_grad_kernel).  No atomics: a repeat gives the same bits.
//
// Precision.  q, k, v and dO are operands as they stand.  What is computed stays fp32 in registers; where it is an operand it is the sum of two or three
// values of 16 bits, in two to six products.  Forward without last states: two of the type (16 bits of a bf16 pair, 22 of a half pair), since what comes of
// them is rounded to the type.  The last states are fp32, and dg and dbeta are what is left of larger terms: with bf16 pairs throughout these were off by up to
// 5.2e-6 and 1.5e-5 of their norms.  So where last states are wanted, and backward, the walks take half pairs for bf16 too (keys and queries as halves times
// a power of two that prep finds, computed values times one per column, so that no size of state or gradient leaves a half's range), and a chunk's
// gradients three bf16, which are an fp32, of S, dS, U and Y: 3e-7 and 1.2e-6, for 15 us in 104 and 8 in 112 (gradients; 4096 tokens, 16 heads, head
// widths of 128).  What only goes into dq and dk, which are rounded to 16 bits, stays pairs.  fp32: v_mfma_f32_16x16x4, no pairs.
// The halves of T, keys and queries have no unit of their own per token: where the keys of a chunk differ in length by a factor of r, |T_ij| is up to
// 2 |k_j| / |k_i|, which half holds for r up to 2^14, and results lose up to log2 r bits (r = 8, 64, 1024, 8192: ht off by 4.6e-7, 2.2e-6, 3.3e-5, 3e-4 of its norm).
#pragma once
#include "attention_docs_tiles.h"

namespace zs {
namespace {

constexpr int DELTA_C = DELTA_CHUNK;
constexpr float DELTA_FORGETS = -200.f;   // log2 of a decay that fp32 does not tell from 0; lower ones, -inf among them, count as this
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// Operands of products of 16 x 16 results over 32 terms: a lane holds 8 values of row (or column) lane % 16, the terms 4 (lane/16) + {0 .. 3, 16 .. 19}:
// the order in which two results above one another, whose rows are 4 (lane/16) + {0 .. 3}, lie in a lane's registers.
template <typename E> struct Op8 { typedef E type __attribute__((ext_vector_type(8))); };
template <typename E> using op8 = typename Op8<E>::type;
__device__ __forceinline__ f32x4 mma1(op8<bf16> a, op8<bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma1(op8<f16> a, op8<f16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma1(op8<float> a, op8<float> b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}
// A value as one operand, or as the sum of two or three, each of what the ones before leave.  Products smaller than the last terms' are left out; small ones
// come first.
template <typename E, int TERMS> struct Opnd { op8<E> t[TERMS]; };
template <typename E, int A, int B> __device__ __forceinline__ f32x4 mma(const Opnd<E, A>& a, const Opnd<E, B>& b, f32x4 c) {
  constexpr int MOST = A > B ? A : B;
#pragma unroll
  for (int order = MOST - 1; order >= 0; --order)
#pragma unroll
    for (int i = A - 1; i >= 0; --i)
      if (i <= order && order - i < B) c = mma1(a.t[i], b.t[order - i], c);
  return c;
}
template <typename M> constexpr int PAIR = sizeof(M) == 2 ? 2 : 1;
template <typename M> using Pair = Opnd<M, PAIR<M>>;
// bf16: both of two values at once, six instructions.
__device__ __forceinline__ void split_two(float x, float y, unsigned& hi, unsigned& lo) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  union { bf16x2 v; unsigned w; } h, l;
  h.v = __builtin_convertvector(f32x2{x, y}, bf16x2);
  l.v = __builtin_convertvector(f32x2{x - __uint_as_float(h.w << 16), y - __uint_as_float(h.w & 0xffff0000u)}, bf16x2);
  hi = h.w;
  lo = l.w;
}
typedef f16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void split_two(float x, float y, f16x2& hi, f16x2& lo) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  hi = __builtin_convertvector(f32x2{x, y}, f16x2);
  lo = __builtin_convertvector(f32x2{x - (float)hi[0], y - (float)hi[1]}, f16x2);
}
template <typename M> __device__ __forceinline__ Pair<M> pair_of(const f32x4& a, const f32x4& b) {
  Pair<M> o;
  if constexpr (__is_same(M, bf16)) {
    union { u32x4 w; op8<bf16> v; } h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4& x = e < 2 ? a : b;
      unsigned hi, lo;
      split_two(x[2 * (e & 1)], x[2 * (e & 1) + 1], hi, lo);
      h.w[e] = hi;
      l.w[e] = lo;
    }
    o.t[0] = h.v;
    o.t[1] = l.v;
  } else if constexpr (__is_same(M, f16)) {
    union { f16x2 w[4]; op8<f16> v; } h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4& x = e < 2 ? a : b;
      split_two(x[2 * (e & 1)], x[2 * (e & 1) + 1], h.w[e], l.w[e]);
    }
    o.t[0] = h.v;
    o.t[1] = l.v;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = e < 4 ? a[e & 3] : b[e & 3];
      o.t[0][e] = from_f<M>(x);
      if constexpr (PAIR<M> == 2) o.t[1][e] = from_f<M>(fp32_value(x - (float)o.t[0][e]));
    }
  }
  return o;
}
template <typename M, int TERMS> __device__ __forceinline__ Opnd<M, TERMS> terms_of(f32x4 a, f32x4 b) {   // bf16: three terms are an fp32
  Opnd<M, TERMS> o;
  if constexpr (TERMS == 1) o.t[0] = pair_of<M>(a, b).t[0];
  else {
    const Pair<M> p = pair_of<M>(a, b);
    o.t[0] = p.t[0];
    o.t[1] = p.t[1];
#pragma unroll
    for (int e = 0; e < 8; ++e) o.t[2][e] = (M)((e < 4 ? a[e & 3] : b[e & 3]) - (float)p.t[0][e] - (float)p.t[1][e]);
  }
  return o;
}

// Sums over the lanes that share lane % 16, and over those that share lane / 16, without LDS.
__device__ __forceinline__ float rows_sum(float x) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float rows_max(float x) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
template <int CTRL> __device__ __forceinline__ float dpp(float x) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true)); }
template <int CTRL> __device__ __forceinline__ unsigned dpp(unsigned x) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ float columns_sum(float x) {
  x += dpp<0xb1>(x);    // neighbours
  x += dpp<0x4e>(x);    // pairs
  x += dpp<0x141>(x);   // the two quads of eight lanes
  return x + dpp<0x140>(x);
}

__device__ __forceinline__ unsigned wave_most(unsigned x) {
  x = max(x, dpp<0xb1>(x));
  x = max(x, dpp<0x4e>(x));
  x = max(x, dpp<0x141>(x));
  x = max(x, dpp<0x140>(x));
  auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  x = max(a[0], a[1]);
  auto b = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return max(b[0], b[1]);
}

// What walks whose states are results, and a chunk's own matrices for them, are computed in: bf16 as half.
template <typename E> struct WalkOf { typedef E type; };
template <> struct WalkOf<bf16> { typedef f16 type; };

// Half: the power of two that brings the largest of a column's values, which lie in the four lanes that share lane % 16, to 2^13 .. 2^14; else 1.
template <typename M, int N> __device__ __forceinline__ float column_unit(const f32x4 (&x)[N]) {
  if constexpr (!__is_same(M, f16)) return 1.f;
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) m = fmaxf(m, fabsf(x[i][r]));
  m = rows_max(m);
  const int e = (int)(__float_as_uint(m) >> 23) & 255;
  return m > 0.f && e < 255 ? __uint_as_float((unsigned)min(max(127 + 13 + 127 - e, 1), 253) << 23) : 1.f;
}
template <typename M> __device__ __forceinline__ float inverse_unit(float unit) {   // of a power of two: exact
  if constexpr (!__is_same(M, f16)) return 1.f;
  return __uint_as_float((254u << 23) - __float_as_uint(unit));
}
template <typename M, int N> __device__ __forceinline__ void pairs_of(Pair<M> (&o)[N / 2], const f32x4 (&x)[N], float unit) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    if constexpr (__is_same(M, f16)) o[i] = pair_of<M>(x[2 * i] * unit, x[2 * i + 1] * unit);
    else o[i] = pair_of<M>(x[2 * i], x[2 * i + 1]);
  }
}

// Places of operands in a tile of rows (Tile: rows come straight from memory, pieces of 16 bytes changed about).
template <typename E, int D> struct TileOps {
  typedef Tile<E, D> TL;
  __device__ __forceinline__ TileOps() {}
  static constexpr int SZ = TL::SZ, OCTET = TL::OCTET;
  unsigned row_[SZ == 4 ? 2 : 4], col_[SZ == 4 ? 8 : 4];
  __device__ __forceinline__ TileOps(unsigned base, int lane) {
    const int g = lane >> 4, i = lane & 15;
#pragma unroll
    for (int p = 0; p < (SZ == 4 ? 2 : 4); ++p)
      row_[p] = base + (i >> 3) * OCTET + (SZ == 4 ? TL::place(i & 7, 4 * p + g) : TL::place(i & 7, 2 * p + (g >> 1)) + 8 * (g & 1));
    if constexpr (SZ == 4) {
#pragma unroll
      for (int p = 0; p < 8; ++p) col_[p] = base + (g >> 1) * OCTET + TL::place(4 * (g & 1) + (p & 3), 4 * (p >> 2) + (i >> 2)) + 4 * (i & 3);
    } else {
#pragma unroll
      for (int p = 0; p < 4; ++p) col_[p] = base + (g >> 1) * OCTET + TL::place(4 * (g & 1) + (i >> 2), 2 * p + ((i & 3) >> 1)) + 8 * (i & 1);
    }
  }
  // row 16 m + lane % 16, columns 32 s + ..
  __device__ __forceinline__ Opnd<E, 1> row(unsigned tile, int m, int s) const {
    Opnd<E, 1> o;
    if constexpr (SZ == 4) {
      const unsigned at = tile + m * 2 * OCTET + s * 1024;
      union { f32x4 h[2]; op8<E> v; } u;
      u.h[0] = lds_read<f32x4>(row_[0] + at);
      u.h[1] = lds_read<f32x4>(row_[1] + at);
      o.t[0] = u.v;
    } else {
      const unsigned at = tile + m * 2 * OCTET + (s >> 1) * 1024;
      union { u32x2 h[2]; op8<E> v; } u;
      u.h[0] = lds_read<u32x2>(row_[2 * (s & 1)] + at);
      u.h[1] = lds_read<u32x2>(row_[2 * (s & 1) + 1] + at);
      o.t[0] = u.v;
    }
    return o;
  }
  // column 16 b + lane % 16, rows 32 s + ..
  __device__ __forceinline__ Opnd<E, 1> column(unsigned tile, int b, int s) const {
    Opnd<E, 1> o;
    if constexpr (SZ == 4) {
      const unsigned at = tile + s * 4 * OCTET + (b >> 1) * 1024;
#pragma unroll
      for (int e = 0; e < 8; ++e) o.t[0][e] = lds_read<float>(col_[(b & 1) * 4 + (e & 3)] + at + (e >> 2) * 2 * OCTET);
    } else {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const unsigned at = col_[b & 3] + tile + s * 4 * OCTET + (b >> 2) * 1024;
      union { s16x4 h[2]; op8<E> v; } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)at);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(at + 2 * OCTET));
      o.t[0] = u.v;
    }
    return o;
  }
  // The same with the 32 columns of a block in another order, in which a row operand's lie together: lane group g has 8 g .. 8 g + 7, so that row
  // 4 g + r of the even (odd) one of two results above one another is the block's 8 g + r (8 g + 4 + r): state_row.
  unsigned srow_[2], scol_[SZ == 4 ? 8 : 2];
  __device__ __forceinline__ void state_places(unsigned base, int lane) {
    const int g = lane >> 4, i = lane & 15;
#pragma unroll
    for (int p = 0; p < 2; ++p) srow_[p] = base + (i >> 3) * OCTET + (SZ == 4 ? TL::place(i & 7, 2 * g + p) : TL::place(i & 7, 4 * p + g));
#pragma unroll
    for (int p = 0; p < (SZ == 4 ? 8 : 2); ++p)
      scol_[p] = base + (g >> 1) * OCTET + (SZ == 4 ? TL::place(4 * (g & 1) + (p & 3), 2 * (i >> 2) + (p >> 2)) + 4 * (i & 3)
                                                    : TL::place(4 * (g & 1) + (i >> 2), 4 * p + (i & 3)));
  }
  // row 16 m + lane % 16, columns of block s
  __device__ __forceinline__ Opnd<E, 1> state_row(unsigned tile, int m, int s) const {
    Opnd<E, 1> o;
    if constexpr (SZ == 4) {
      const unsigned at = tile + m * 2 * OCTET + s * 1024;
      union { f32x4 h[2]; op8<E> v; } u;
      u.h[0] = lds_read<f32x4>(srow_[0] + at);
      u.h[1] = lds_read<f32x4>(srow_[1] + at);
      o.t[0] = u.v;
    } else o.t[0] = lds_read<op8<E>>(srow_[s & 1] + tile + m * 2 * OCTET + (s >> 1) * 1024);
    return o;
  }
  // result b's row lane % 16 of the columns, rows 32 s + ..
  __device__ __forceinline__ Opnd<E, 1> state_column(unsigned tile, int b, int s) const {
    Opnd<E, 1> o;
    if constexpr (SZ == 4) {
      const unsigned at = tile + s * 4 * OCTET + (b >> 1) * 1024;
#pragma unroll
      for (int e = 0; e < 8; ++e) o.t[0][e] = lds_read<float>(scol_[(b & 1) * 4 + (e & 3)] + at + (e >> 2) * 2 * OCTET);
    } else {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const unsigned at = scol_[(b >> 1) & 1] + tile + s * 4 * OCTET + (b >> 2) * 1024 + 8 * (b & 1);
      union { s16x4 h[2]; op8<E> v; } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)at);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(at + 2 * OCTET));
      o.t[0] = u.v;
    }
    return o;
  }
  __device__ __forceinline__ void move_state_places(unsigned by) {
#pragma unroll
    for (int p = 0; p < 2; ++p) srow_[p] += by;
#pragma unroll
    for (int p = 0; p < (SZ == 4 ? 8 : 2); ++p) scol_[p] += by;
  }
  // row 16 m + lane % 16, columns 16 b + 4 (lane/16) ..
  __device__ __forceinline__ f32x4 quad(unsigned tile, int m, int b) const {
    f32x4 o;
    if constexpr (SZ == 4) o = lds_read<f32x4>(row_[b & 1] + tile + m * 2 * OCTET + (b >> 1) * 1024);
    else {
      typedef E quad_t __attribute__((ext_vector_type(4)));
      const quad_t q = lds_read<quad_t>(row_[b & 3] + tile + m * 2 * OCTET + (b >> 2) * 1024);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (float)q[e];
    }
    return o;
  }
};

// What delta_prep_kernel leaves of a chunk and value head: per token exp(G), exp(G_last - G), beta, and exp(G_last) in the fourth row's first place,
// behind it what undoes the units of keys and queries;
// then matrices as operands, pair by pair: of T and P, lower triangles, rows by m and terms by s <= m/2; of T^T and P^T, upper ones, s >= m/2.
constexpr int REC_GATES = 1024, REC_OP = 2048, REC_TRIANGLE = 6 * REC_OP;
constexpr int REC_T = REC_GATES, REC_P = REC_T + REC_TRIANGLE, REC_FWD = REC_P + REC_TRIANGLE;
constexpr int REC_TT = REC_P + REC_TRIANGLE, REC_G = REC_TT + REC_TRIANGLE, REC_BWD = REC_G + 512;   // backward: P^T in the place of P; G, 64 bits
static_assert(REC_FWD == DELTA_RECORD_FWD && REC_BWD == DELTA_RECORD_BWD, "");
__device__ __forceinline__ constexpr int lower_op(int m, int s) { return m < 2 ? m : 2 + (m - 2) * 2 + s; }
__device__ __forceinline__ constexpr int upper_op(int m, int s) { return m < 2 ? 2 * m + s : 4 + (m - 2); }
template <typename M> __device__ __forceinline__ void store_op(char* to, const Pair<M>& o, int lane) {
  if constexpr (sizeof(M) == 4) {
    union { op8<M> v; f32x4 h[2]; } u;
    u.v = o.t[0];
    reinterpret_cast<f32x4*>(to)[lane] = u.h[0];
    reinterpret_cast<f32x4*>(to)[64 + lane] = u.h[1];
  } else {
    reinterpret_cast<op8<M>*>(to)[lane] = o.t[0];
    reinterpret_cast<op8<M>*>(to)[64 + lane] = o.t[1];
  }
}
template <typename M> __device__ __forceinline__ Pair<M> load_op(unsigned lds_of_lane) {   // 16 lane bytes behind the operand's begin
  Pair<M> o;
  if constexpr (sizeof(M) == 4) {
    union { op8<M> v; f32x4 h[2]; } u;
    u.h[0] = lds_read<f32x4>(lds_of_lane);
    u.h[1] = lds_read<f32x4>(lds_of_lane + 1024);
    o.t[0] = u.v;
  } else {
    o.t[0] = lds_read<op8<M>>(lds_of_lane);
    o.t[1] = lds_read<op8<M>>(lds_of_lane + 1024);
  }
  return o;
}
// Loads into LDS that run ahead.  The compiler waits for all of those that it knows of before the next transposing read, whatever that reads; these it
// does not know, and the waits are the callers' (tile_wait before the barrier that publishes them).  64 times 16 bytes, from the
// lanes' offsets behind `base`, of which `bytes` may be read (zeros behind them), to `lds` on.
// RUN > 1: as many times, 1 KB on in both places, by offsets of the instructions.
template <int RUN = 1> __device__ __forceinline__ void load_ahead(unsigned lds, const void* base, int bytes, unsigned offset) {
  const uint64_t at = (uint64_t)(uintptr_t)base;
  u32x4 rs;
  rs[0] = __builtin_amdgcn_readfirstlane((unsigned)at);
  rs[1] = __builtin_amdgcn_readfirstlane((unsigned)(at >> 32) & 0xffffu);
  rs[2] = __builtin_amdgcn_readfirstlane((unsigned)bytes);
  rs[3] = 0x00020000u;
  static_assert(RUN == 1 || RUN == 2 || RUN == 4, "");
  unsigned m0;   // as it was: the compiler may have a use for it
  if constexpr (RUN == 1)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(rs) : "memory");
  else if constexpr (RUN == 2)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %2, %3, 0 offen offset:0x400 lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(rs) : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %2, %3, 0 offen offset:0x400 lds\n\tbuffer_load_dwordx4 %2, %3, 0 offen offset:0x800 lds\n\t"
                 "buffer_load_dwordx4 %2, %3, 0 offen offset:0xc00 lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(rs) : "memory");
}
template <typename E, int D, int ROWS, int NW> __device__ __forceinline__ void tile_ahead(const TileLoad<E, D, ROWS, NW>& t, unsigned lds, const E* head, int row0, int end, int wave) {
  typedef Tile<E, D> TL;
  const int rows = min(end - row0, ROWS), bytes = rows > 0 ? (rows - 1) * t.ld * TL::SZ + t.width : 0;
#pragma unroll
  for (int i = 0; i < TileLoad<E, D, ROWS, NW>::N; ++i) {
    const int sq = wave + NW * i, oct = sq / TL::SQUARES, q = sq % TL::SQUARES;
    unsigned from = t.at[0];
#pragma unroll
    for (int k = 1; k < TL::SQUARES; ++k) from = q == k ? t.at[k] : from;
    load_ahead(lds + oct * TL::OCTET + q * 1024, head + (int64_t)row0 * t.ld, bytes, from + (unsigned)(8 * oct * t.ld * TL::SZ));
  }
}
// Waits until at most N of a wave's loads and stores are under way: all but its last N.
template <int N> __device__ __forceinline__ void loads_but() {
  static_assert(N < 64, "");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
  __builtin_amdgcn_sched_barrier(0);
}
// KB times 1024 bytes that lie together, as they are, by NW waves, KB / NW loads each.
template <int KB, int NW> __device__ __forceinline__ void bytes_ahead(unsigned lds, const char* from, int wave, int lane) {
  constexpr int RUN = KB % (4 * NW) == 0 ? 4 : KB % (2 * NW) == 0 ? 2 : 1;
  static_assert(KB % (RUN * NW) == 0, "");
#pragma unroll
  for (int i = 0; i < KB / RUN / NW; ++i) {
    const unsigned at = (unsigned)(wave + NW * i) * (RUN * 1024);
    load_ahead<RUN>(lds + at, from, KB * 1024, at + 16 * lane);
  }
}

// A tile of 64 rows whose squares lie in order.
template <typename TL, int NW> __device__ __forceinline__ void squares_ahead(unsigned lds, const void* from, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < 8 / NW; ++i) {
    const int oct = wave + NW * i;
    load_ahead<TL::SQUARES>(lds + oct * TL::OCTET, from, 8 * TL::SQUARES * 1024, (unsigned)(oct * TL::SQUARES * 1024 + 16 * lane));
  }
}

// ------------------------------------------------------------------------------------------ a chunk's own matrices
constexpr int TRI_LD = 68;   // floats of a row of a 64 x 64 matrix in LDS: rows 16 bytes aligned, four banks apart
// T = (1 + A)^-1 of a strictly lower A, both in LDS, by four waves.  Blocks of 16 on the diagonal by substitution, four rows at a time, by the lanes that hold
// them, and what these leave of the others by a product; then block by block away from it, T_ij = -T_ii (sum over k of A_ik T_kj), in fp32 products.  Every
// step solves for values of T itself, which are bounded where the rule is stable; powers of A, which are not, do not occur.
__device__ __forceinline__ void invert_lower(const float* A, float* T, int wave, int lane) {
  const int g = lane >> 4, c = lane & 15;
  {
    const float* block = A + (16 * wave) * TRI_LD + 16 * wave;
    const f32x4 column = *reinterpret_cast<const f32x4*>(block + c * TRI_LD + 4 * g);   // of row c
    f32x4 own[4], x;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      own[r] = *reinterpret_cast<const f32x4*>(block + (4 * g + r) * TRI_LD + 4 * g);
      x[r] = 4 * g + r == c ? 1.f : 0.f;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bool now = g == q;
      f32x4 y = x;
#pragma unroll
      for (int r = 1; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < r; ++e) y[r] = fmaf(-own[r][e], y[e], y[r]);
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = now ? y[r] : x[r];
      x = y;
      if (q < 3) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(now ? -column[e] : 0.f, now ? y[e] : 0.f, x, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = now ? y[r] : x[r];
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) T[(16 * wave + 4 * g + r) * TRI_LD + 16 * wave + c] = x[r];
  }
#pragma unroll
  for (int d = 1; d < 4; ++d) {
    __syncthreads();
    const int i = wave, j = wave - d;
    if (j >= 0) {
      f32x4 x[3] = {};   // a sum of its own for each block, so that none waits for another
      const f32x4 t = *reinterpret_cast<const f32x4*>(T + (16 * i + c) * TRI_LD + 16 * i + 4 * g);
#pragma unroll
      for (int k = 0; k < d; ++k) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(A + (16 * i + c) * TRI_LD + 16 * (j + k) + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], T[(16 * (j + k) + 4 * g + e) * TRI_LD + 16 * j + c], x[k], 0, 0, 0);
      }
      const f32x4 sum = d == 1 ? x[0] : d == 2 ? x[0] + x[1] : x[0] + x[1] + x[2];
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) y = __builtin_amdgcn_mfma_f32_16x16x4f32(t[e], sum[e], y, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) T[(16 * i + 4 * g + r) * TRI_LD + 16 * j + c] = -y[r];
    }
  }
  __syncthreads();
}

// The running sum of a chunk's log2 decays in 64 bits: sums of many small and a few large ones, of which small differences are wanted.
__device__ __forceinline__ double running_sum(double x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}
__device__ __forceinline__ float decay(double to, double from) { return __builtin_amdgcn_exp2f((float)(to - from)); }

// Rows of the table.  Whatever it holds, they lie inside the tokens, chunks and documents.
struct ChunkRow { int first, count; };
__device__ __forceinline__ ChunkRow chunk_row(const DeltaRule& a, int c) {
  const int4 r = reinterpret_cast<const int4*>(a.chunks)[1 + a.ndocs + c];
  const int first = min(max(r.x, 0), a.T);
  return ChunkRow{first, min(max(r.y, 0), min(DELTA_C, a.T - first))};
}
struct DocRow { int first, count, chunk0, doc; };
__device__ __forceinline__ DocRow doc_row(const DeltaRule& a, int rank) {
  const int4 r = reinterpret_cast<const int4*>(a.chunks)[1 + rank];
  const int first = min(max(r.x, 0), a.T), chunk0 = min(max(r.z, 0), a.nchunks);
  return DocRow{first, min(min(max(r.y, 0), a.T - first), (a.nchunks - chunk0) * DELTA_C), chunk0, min(max(r.w, 0), a.ndocs - 1)};
}

// Rows of no document become zeros: the last DELTA_FILL blocks of a grid of chunks share them.
template <typename E> __device__ __forceinline__ void fill_rows(E* p, int64_t ld, int width, int T, int begin, int end, int block) {
  const int rows = begin + (T - end), vecs = width / Vec<E>::N;
  for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < (int64_t)rows * vecs; i += DELTA_FILL * 256) {
    const int r = (int)(i / vecs), t = r < begin ? r : end + (r - begin);
    *reinterpret_cast<typename Vec<E>::type*>(p + t * ld + (i % vecs) * Vec<E>::N) = typename Vec<E>::type{};
  }
}

// A workgroup per chunk and key head; the value heads of the key head one after the other: K K^T and Q K^T are formed once for them.  Bound by phases that follow
// one another, of which four workgroups on a CU hide a part; of 17600 cycles 3500 until keys and queries are there, 4300 their products, 3900 A and P, 4000 the
// inverse (5500 with a lane per column and row after row in its diagonal blocks).  4096 tokens of 16 heads of 128 19.5 us, 25 with what the gradients take
// besides (they write 28 and 42 MB, 6 and 9 us at the rate of a large copy).
constexpr int prep_lds(int tile) { return 2 * tile > 2 * 64 * TRI_LD * 4 ? 2 * tile : 2 * 64 * TRI_LD * 4; }   // A and T take the place of keys and queries
template <typename E, int DK> constexpr int PREP_LDS = prep_lds(Tile<E, DK>::bytes(DELTA_C));
template <typename E, int DK> constexpr int PREP_GROUPS = PREP_LDS<E, DK> <= 36 * 1024 ? 4 : 2;   // on a CU
template <typename E, typename A16, int DK, bool BWD> __global__ __launch_bounds__(256, (PREP_GROUPS<E, DK>)) void delta_prep_kernel(DeltaRule a) {
  typedef Tile<E, DK> TL;
  constexpr int TILE = TL::bytes(DELTA_C), KS = DK / 32;
  __shared__ __align__(16) char tiles[PREP_LDS<E, DK>];
  float *A = reinterpret_cast<float*>(tiles), *Tm = A + 64 * TRI_LD;
  __shared__ double G[64];
  __shared__ float B[64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, i16 = lane & 15;
  const int kv = blockIdx.y, group = a.nv / a.nk;
  if ((int)blockIdx.x >= a.nchunks) {
    const int4 head = *reinterpret_cast<const int4*>(a.chunks);
    const int begin = min(max(head.y, 0), a.T), end = min(max(head.z, begin), a.T), block = (int)blockIdx.x - a.nchunks;
    if constexpr (BWD) {
      fill_rows((E*)a.dq + kv * a.dk, a.lddq, a.dk, a.T, begin, end, block);
      fill_rows((E*)a.dkey + kv * a.dk, a.lddk, a.dk, a.T, begin, end, block);
      fill_rows((E*)a.dval + kv * group * a.dv, a.lddv, group * a.dv, a.T, begin, end, block);
      for (int i = block * 256 + threadIdx.x; i < begin + (a.T - end); i += DELTA_FILL * 256) {
        const int t = i < begin ? i : end + (i - begin);
        for (int h = 0; h < group; ++h) a.dg[(int64_t)t * a.nv + kv * group + h] = a.dbeta[(int64_t)t * a.nv + kv * group + h] = 0.f;
      }
    } else fill_rows((E*)a.o + kv * group * a.dv, a.ldo, group * a.dv, a.T, begin, end, block);
    return;
  }
  const ChunkRow c = chunk_row(a, blockIdx.x);
  if (c.count <= 0) return;
  const unsigned smem = lds_address(tiles);
  const bool in = lane < c.count;   // the first wave's token, and its gates; before keys and queries, since loads come back in order
  const int64_t first_gate = (int64_t)(c.first + (in ? lane : 0)) * a.nv + kv * group;
  float g_in = a.g[first_gate], beta_in = a.beta[first_gate];
  __builtin_amdgcn_sched_barrier(0);
  {
    const TileLoad<E, DK, DELTA_C, 4> load_k(a.ldk, lane, a.dk), load_q(a.ldq, lane, a.dk);
    load_k.fetch(smem, (const E*)a.k + kv * a.dk, c.first, c.first + c.count, wave);
    load_q.fetch(smem + TILE, (const E*)a.q + kv * a.dk, c.first, c.first + c.count, wave);
  }
  // A head's gates, by the first wave: the first head's while keys and queries are under way (after them: 3700 of 17700 cycles).
  auto gates_of = [&](int h) {
    char* rec = a.records + ((int64_t)blockIdx.x * a.nv + h) * (BWD ? REC_BWD : REC_FWD);
    const float gl = in ? g_in * 1.4426950408889634f : 0.f, beta = in ? beta_in : 0.f;
    const double sum = running_sum((double)(gl < DELTA_FORGETS ? DELTA_FORGETS : gl), lane), last = __shfl(sum, 63, 64);
    G[lane] = sum;
    B[lane] = beta;
    float* gates = reinterpret_cast<float*>(rec);
    gates[lane] = in ? decay(sum, 0.0) : 0.f;
    gates[64 + lane] = in ? decay(last, sum) : 0.f;
    gates[128 + lane] = beta;
    if (lane == 0) gates[192] = decay(last, 0.0);
    if constexpr (BWD) reinterpret_cast<double*>(rec + REC_G)[lane] = sum;
  };
  if (wave == 0) gates_of(kv * group);
  tile_wait();
  __syncthreads();
  const TileOps<E, DK> at(smem, lane);
  float k_unit = 1.f, q_unit = 1.f;
  if constexpr (!__is_same(A16, E)) {   // keys and queries as halves, times powers of two that bring the largest of either to 2^3 .. 2^4
    constexpr int PIECES = DK / 8, MINE = 64 * PIECES / 256;
    typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
    __shared__ unsigned most_of[2][4];
    bf16x8 x[2][MINE];
    unsigned most[2];   // of the bits below the sign, which compare as the values do
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      u16x8 m = {};
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        const int piece = (int)threadIdx.x + 256 * i, row = piece / PIECES, p = piece % PIECES;
        const u16x8 bits = lds_read<u16x8>(smem + t * TILE + row / 8 * TL::OCTET + (p >> 3) * 1024 + TL::place(row & 7, p & 7));
        x[t][i] = __builtin_bit_cast(bf16x8, bits);
        m = __builtin_elementwise_max(m, bits & (unsigned short)0x7fff);
      }
      most[t] = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) most[t] = max(most[t], (unsigned)m[e]);
      most[t] = wave_most(most[t]);
      if (lane == 0) most_of[t][wave] = most[t];
    }
    __syncthreads();
    auto unit = [&](int t) {
      const unsigned m = max(max(most_of[t][0], most_of[t][1]), max(most_of[t][2], most_of[t][3]));
      const int e = (int)(m >> 7);
      return m > 0 && e < 255 ? __uint_as_float((unsigned)min(max(257 - e, 77), 177) << 23) : 1.f;
    };
    k_unit = unit(0);
    q_unit = unit(1);
    f16* to = a.halves + ((int64_t)blockIdx.x * a.nk + kv) * (2 * 64 * DK);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        f16x8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = (f16)((float)x[t][i][e] * (t ? q_unit : k_unit));
        const int piece = (int)threadIdx.x + 256 * i, row = piece / PIECES, p = piece % PIECES;   // squares as they will lie in LDS
        *reinterpret_cast<f16x8*>(to + t * 64 * DK + (row / 8 * TL::SQUARES + (p >> 3)) * 512 + TL::place(row & 7, p & 7) / 2) = h;
      }
  }
  const float p_unit = k_unit * q_unit, k_inv = 1.f / k_unit, q_inv = 1.f / q_unit;   // powers of two
  // This wave's rows (kk, and qk of P^T backward: rows j) or columns (qk of P: rows of P^T are keys) against all tiles of the other side.  Of triangles, so that
  // its columns of P are from the other end.
  const int pw = BWD ? wave : 3 - wave;
  f32x4 kk[4], qk[4];
#pragma unroll
  for (int n = 0; n < 4; ++n) kk[n] = qk[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const Opnd<E, 1> mine = at.row(0, wave, s), q_mine = at.row(TILE, pw, s);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const Opnd<E, 1> k_n = at.row(0, n, s);
      if (n <= wave) kk[n] = mma(mine, k_n, kk[n]);                                     // rows i of this wave, columns j of tile n
      if constexpr (BWD) {
        if (n >= wave) qk[n] = mma(at.row(TILE, n, s), mine, qk[n]);                    // rows i of tile n, columns j of this wave
      } else if (n <= pw) qk[n] = mma(k_n, q_mine, qk[n]);                              // rows j of tile n, columns i of this wave
    }
  }
  for (int hg = 0; hg < group; ++hg) {
    const int h = kv * group + hg;
    char* rec = a.records + ((int64_t)blockIdx.x * a.nv + h) * (BWD ? REC_BWD : REC_FWD);
    __syncthreads();   // the head before, or keys and queries, are done with the LDS
    if (wave == 0 && hg > 0) {
      g_in = a.g[first_gate + hg];
      beta_in = a.beta[first_gate + hg];
      gates_of(h);
    }
    if (wave == 0 && lane < 2) reinterpret_cast<float*>(rec)[193 + lane] = lane ? q_inv : k_inv;
    if (hg > 0) __syncthreads();
    {   // A
      double gi[4];
      float bi[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        gi[r] = G[16 * wave + 4 * g + r];
        bi[r] = B[16 * wave + 4 * g + r];
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const double gj = G[16 * n + i16];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int i = 16 * wave + 4 * g + r, j = 16 * n + i16;
          if (n <= wave) A[i * TRI_LD + j] = j < i ? bi[r] * decay(gi[r], gj) * kk[n][r] : 0.f;
          if (n > wave) Tm[i * TRI_LD + j] = 0.f;
        }
      }
    }
    // P: tiles as they lie, two of them an operand
    f32x4 p[4];
    const double gc = G[16 * pw + i16];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * n + 4 * g + r, col = 16 * pw + i16;
        const double gr = G[row];
        if constexpr (BWD) p[n][r] = row >= col ? p_unit * qk[n][r] * decay(gr, gc) : 0.f;   // P_row,col
        else p[n][r] = row <= col ? p_unit * qk[n][r] * decay(gc, gr) : 0.f;                 // P_col,row
      }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if constexpr (BWD) {
        if (2 * s + 1 >= wave) store_op<A16>(rec + REC_P + upper_op(wave, s) * REC_OP, pair_of<A16>(p[2 * s], p[2 * s + 1]), lane);
      } else if (2 * s <= pw) store_op<A16>(rec + REC_P + lower_op(pw, s) * REC_OP, pair_of<A16>(p[2 * s], p[2 * s + 1]), lane);
    }
    __syncthreads();
    invert_lower(A, Tm, wave, lane);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (2 * s <= wave) {
        const float* row = Tm + (16 * wave + i16) * TRI_LD + 32 * s + 4 * g;
        store_op<A16>(rec + REC_T + lower_op(wave, s) * REC_OP, pair_of<A16>(*reinterpret_cast<const f32x4*>(row), *reinterpret_cast<const f32x4*>(row + 16)), lane);
      }
      if constexpr (BWD)
        if (2 * s + 1 >= wave) {
          f32x4 x, y;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = Tm[(32 * s + 4 * g + e) * TRI_LD + 16 * wave + i16];
            y[e] = Tm[(32 * s + 16 + 4 * g + e) * TRI_LD + 16 * wave + i16];
          }
          store_op<A16>(rec + REC_TT + upper_op(wave, s) * REC_OP, pair_of<A16>(x, y), lane);
        }
    }
  }
}

// ------------------------------------------------------------------------------------------ from chunk to chunk
// A workgroup walks a document's chunks for one value head and 16 NW columns of its state.  Two waves carry 16 columns of the state, a half of its rows
// each, in their registers, and it never leaves them: a result's registers, two above one another, are the next product's operand.  What a chunk
// waits for is the chain of these waves: K S, a half of the tokens each; what that leaves, Z, exchanged; T Z, by both; K^T of that into the
// own rows; the new state as pairs, exchanged.  All else is done by others: each such pair of waves has two helpers that share out what it does not wait for (T Z
// once more for the results, what the gradients' walk adds to its state, the stores of states and u), with 12 KB of LDS between the four; the loads
// are waves' of their own, or, with 32 columns, where these would be a third wave on a SIMD, the second helpers'.  Two barriers a chunk: the first publishes the
// state, and matrices, values and queries of the chunk, the second Z, and the next chunk's keys.  All of these come straight into LDS, a chunk ahead where
// two of them fit.  What bounds a walk: that chain, 3000 cycles a chunk (1.4 us) of 16 columns alone on a CU, 4100 where two sets of columns and their
// helpers share the SIMDs.  bf16, widths of 128: one document of 8192 tokens, 32 heads over 16, 177 us; 4096 tokens in documents, 16 heads, 47 (with one
// helper, and more to load in one phase than in the other: 188 and 53), and both walks of their gradients 110: 7900 cycles a chunk, in which the helpers are
// what the others wait for (2000 to 3700 cycles for what a gradient gets from Q and dO, as long for the stores of states and y).
enum DeltaWalk { WALK_RESULTS = 0, WALK_STATES = 1, WALK_GRADIENTS = 2 };   // o and the last state; the states and u for the gradients; the states' gradients and y
constexpr int HELPERS = 2;                                       // of 16 columns
constexpr int walk_loaders(int NW) { return NW == 1 ? 4 : 0; }   // waves that only load; to ask for 1 KB takes a wave 50 to 70 cycles
constexpr int walk_threads(int NW) { return 64 * ((2 + HELPERS) * NW + walk_loaders(NW)); }
template <int V> struct Int { static constexpr int value = V; };

template <typename E, typename M, int DK, int NW, int KIND> struct WalkLds {
  typedef Tile<M, DK> TL;
  typedef Tile<E, 64> VL;
  static constexpr int REC = KIND == WALK_STATES ? REC_P : REC_FWD;   // gates and T; and P; or gates, P^T and T^T
  static constexpr int VSIZE = VL::bytes(DELTA_C), QSIZE = KIND == WALK_STATES ? 0 : TL::bytes(DELTA_C);
  static constexpr int HAND = DK * 64 + 4096 + (KIND == WALK_GRADIENTS ? DK * 64 : 0);   // of 16 columns: the state as pairs (fp32: as it is); Z; what is added to it
  static constexpr int FIRST = TL::bytes(DELTA_C) + REC, SECOND = VSIZE + QSIZE, ROOM = 160 * 1024 - NW * HAND;
  // Two buffers of all a chunk brings, or of its keys and matrices, or one.
  static constexpr int NBUF = 2 * FIRST + SECOND <= ROOM ? 2 : 1, VBUF = 2 * (FIRST + SECOND) <= ROOM ? 2 : 1;
  static constexpr int K = 0, R = TL::bytes(DELTA_C), V = NBUF * FIRST, Q = V + VSIZE, H = V + VBUF * SECOND, BYTES = H + NW * HAND;
  // Half's units, in the gaps of 128 bytes behind octets of the first keys.  Of set n of 16 columns: behind octet n those of the state, of its two halves of
  // rows 64 bytes each; behind octet 4 + n those of Z, of its two halves of tokens.
  static constexpr int UNITS = TL::OCTET - 128, UNITS_Z = 4 * TL::OCTET;
  static_assert(NW <= 4 && TL::OCTET - 128 >= TL::SQUARES * 1024 && TL::bytes(DELTA_C) >= 8 * TL::OCTET, "");
  static_assert(BYTES <= 160 * 1024, "");
};

// Row of the state that a lane's register r of result i has (lane group g), see TileOps.
__device__ __forceinline__ int state_row(int i, int g, int r) { return 32 * (i >> 1) + 8 * g + 4 * (i & 1) + r; }
template <typename T> __device__ __forceinline__ void lds_write(unsigned at, const T& v) { *(__attribute__((address_space(3))) T*)(uintptr_t)at = v; }
template <typename M> __device__ __forceinline__ void write_op(unsigned lds_of_lane, const Pair<M>& x) {   // as load_op reads it
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    union { op8<M> v; f32x4 h[sizeof(op8<M>) / 16]; } u;
    u.v = x.t[PAIR<M> == 2 ? p : 0];
    lds_write(lds_of_lane + p * 1024, u.h[PAIR<M> == 2 ? 0 : p]);
  }
}

// M: what its products are of.
template <typename E, typename M, int DK, int NW, int KIND> __device__ __forceinline__ void delta_walk(char* smem_raw, const DeltaRule& a, int doc_rank, int h, int c0) {
  typedef WalkLds<E, M, DK, NW, KIND> L;
  constexpr int RT = DK / 16, KS = DK / 32, HT = RT / 2, HS = KS / 2, LOADERS = walk_loaders(NW), FW = LOADERS ? LOADERS : NW;
  constexpr bool HALF_E = __is_same(M, f16), COPIES = !__is_same(M, E), BACK = KIND == WALK_GRADIENTS, RESULTS = KIND == WALK_RESULTS, AHEAD = L::NBUF == 2, ALL_AHEAD = L::VBUF == 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = wave % NW, g = lane >> 4, i16 = lane & 15;
  const bool chain = wave < 2 * NW, loads = wave >= (LOADERS ? 4 : 3) * NW;
  const int fw = wave - (LOADERS ? 4 : 3) * NW;
  const DocRow row = doc_row(a, doc_rank);
  const int first = row.first, count = row.count, chunk0 = row.chunk0, doc = row.doc, chunks = (count + DELTA_C - 1) / DELTA_C;
  const int kv = h / (a.nv / a.nk), w0 = c0 + 16 * mine, col = w0 + i16;    // the wave's first column and the lane's
  const unsigned smem = lds_address(smem_raw), hand = smem + L::H + mine * L::HAND + 16 * lane, hand_z = hand + DK * 64, hand_add = hand_z + 4096;
  const unsigned units = smem + L::UNITS + mine * Tile<M, DK>::OCTET;
  const int step = BACK ? -1 : 1;
  const int64_t states = (int64_t)a.dk * a.dv;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

  // ---- loads
  const TileLoad<E, DK, DELTA_C, FW> load_k(a.ldk, lane, a.dk), load_q(a.ldq, lane, a.dk);
  const TileLoad<E, 64, DELTA_C, FW> load_v(BACK ? a.ldo : a.ldv, lane, min(a.dv - c0, 16 * NW));
  // Loads of a wave, at least: of the keys, of the chunk's matrices, of values and queries.
  constexpr int KEYS = TileLoad<M, DK, DELTA_C, FW>::N, MATS = (L::REC - REC_GATES) / 1024 / FW;
  constexpr int SECOND = TileLoad<E, 64, DELTA_C, FW>::N + (KIND == WALK_STATES ? 0 : TileLoad<M, DK, DELTA_C, FW>::N);
  auto copies = [&](int c) { return a.halves + ((int64_t)(chunk0 + c) * a.nk + kv) * (2 * DELTA_C * DK); };
  auto fetch_keys = [&](int c, unsigned to) {
    const int t0 = first + DELTA_C * c, end = min(first + count, t0 + DELTA_C);
    if constexpr (COPIES) squares_ahead<Tile<M, DK>, FW>(to + L::K, copies(c), fw, lane);
    else tile_ahead(load_k, to + L::K, (const E*)a.k + kv * a.dk, t0, end, fw);
  };
  auto fetch_mats = [&](int c, unsigned to) {
    const char* rec = a.records + ((int64_t)(chunk0 + c) * a.nv + h) * (RESULTS ? REC_FWD : REC_BWD);
    if (fw == 0) load_ahead(to + L::R, rec, REC_GATES, 16 * lane);
    bytes_ahead<(L::REC - REC_GATES) / 1024, FW>(to + L::R + REC_GATES, rec + (BACK ? REC_P : REC_GATES), fw, lane);   // P^T and T^T lie side by side
  };
  auto fetch_second = [&](int c, unsigned by) {
    const int t0 = first + DELTA_C * c, end = min(first + count, t0 + DELTA_C);
    tile_ahead(load_v, smem + L::V + by, (BACK ? (const E*)a.dout : (const E*)a.v) + h * a.dv + c0, t0, end, fw);
    if constexpr (KIND != WALK_STATES) {
      if constexpr (COPIES) squares_ahead<Tile<M, DK>, FW>(smem + L::Q + by, copies(c) + DELTA_C * DK, fw, lane);
      else tile_ahead(load_q, smem + L::Q + by, (const E*)a.q + kv * a.dk, t0, end, fw);
    }
  };
  auto fetch_all = [&](int c) {
    fetch_keys(c, smem);
    fetch_mats(c, smem);
    fetch_second(c, 0);
  };
  int c = BACK ? chunks - 1 : 0;
  if (loads && chunks > 0) {
    fetch_all(c);
    if (AHEAD && chunks > 1) {
      fetch_keys(c + step, smem + L::FIRST);
      if constexpr (ALL_AHEAD) fetch_second(c + step, L::SECOND);
      loads_but<KEYS + (ALL_AHEAD ? SECOND : 0)>();
    } else tile_wait();
  }
  // The two barriers of chunk n, and the loading waves' part of them: what they have to see arrived before, what they ask for behind.  After the second one
  // nothing of the chunk's keys, values and queries is read from LDS any more, and the chunk after the next takes their place; its matrices
  // follow in the next phase, so that a wave has about as much to ask for in either.
  auto begin_chunk = [&](int n) {
    if (AHEAD && loads && n + 1 < chunks) fetch_mats(c + step, smem + ((n + 1) & 1) * L::FIRST);
  };
  auto middle = [&](int n) {
    if (AHEAD && loads && n + 1 < chunks) loads_but<MATS + (ALL_AHEAD ? SECOND : 0)>();   // the next keys
    __syncthreads();
    if (AHEAD && loads && n + 1 < chunks) {
      if constexpr (!ALL_AHEAD) fetch_second(c + step, 0);
      if (n + 2 < chunks) {
        fetch_keys(c + 2 * step, smem + (n & 1) * L::FIRST);
        if constexpr (ALL_AHEAD) fetch_second(c + 2 * step, (n & 1) * L::SECOND);
      }
    }
  };
  auto end_chunk = [&](int n) {
    if (AHEAD && loads) {   // the next matrices, values and queries
      if (n + 2 < chunks) loads_but<KEYS + (ALL_AHEAD ? SECOND : 0)>();
      else tile_wait();
    }
    __syncthreads();
    if constexpr (!AHEAD) {
      if (loads && n + 1 < chunks) {
        fetch_all(c + step);
        tile_wait();
      }
      __syncthreads();
    }
  };

  if (chain) {
    const int half = wave / NW;   // of the state's rows, and of the tokens
    const TileOps<E, 64> at_v(smem + L::V, lane);
    TileOps<M, DK> at;
    at.state_places(smem + L::K, lane);
    // Of keys' rows the columns that belong to this half of the state come first, of their columns only these: either 64 columns, whose places
    // change places, or further ones.
    constexpr bool SWAP = sizeof(E) == 2 && DK == 64;
    if (SWAP && half) {
      const unsigned r0 = at.srow_[0], c0_ = at.scol_[0];
      at.srow_[0] = at.srow_[1];
      at.srow_[1] = r0;
      at.scol_[0] = at.scol_[1];
      at.scol_[1] = c0_;
    }
    const unsigned own = SWAP ? 0u : (unsigned)(half * (sizeof(E) == 2 ? 1024 : HS * 1024)), not_own = SWAP ? 0u : (sizeof(E) == 2 ? 1024u : HS * 1024u) - own;
    const bool live = col < a.dv;
    f32x4 S[HT];
    Pair<M> sp[HS];
    float s_unit = 1.f;
    auto publish_state = [&]() {
      if constexpr (HALF_E) {   // of these rows; the other half's may be another
        s_unit = column_unit<M>(S);
        if (lane < 16) lds_write(units + 64 * half + 4 * lane, s_unit);
      }
      pairs_of<M>(sp, S, s_unit);
#pragma unroll
      for (int s = 0; s < HS; ++s) write_op<M>(hand + (HS * half + s) * 2048, sp[s]);
    };
    const float* from = BACK ? a.dht : a.h0;
#pragma unroll
    for (int i = 0; i < HT; ++i) {
      S[i] = zero;
      if (from)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at_row = state_row(HT * half + i, g, r);
          if (live && at_row < a.dk) S[i][r] = from[((int64_t)doc * a.nv + h) * states + (int64_t)at_row * a.dv + col];
        }
    }
    if (chunks > 0) publish_state();
    __syncthreads();
    Opnd<M, 1> kf[HS][2], ko[HS][2];   // this half's rows of the chunk's keys: of this and of the other half's columns
    auto load_keys = [&]() {
      const unsigned rows = half * 4 * Tile<M, DK>::OCTET;
#pragma unroll
      for (int s = 0; s < HS; ++s)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          kf[s][m] = at.state_row(rows + own, m, s);
          ko[s][m] = at.state_row(rows + not_own, m, SWAP ? 1 : s);
        }
    };
    if (chunks > 0) load_keys();
    for (int n = 0; n < chunks; ++n, c += step) {
      const unsigned buf = AHEAD ? (unsigned)(n & 1) * L::FIRST : 0u, gates = smem + buf + L::R, ops = gates + REC_GATES + 16 * lane, gates4 = gates + 16 * g;
      const unsigned second = ALL_AHEAD ? (unsigned)(n & 1) * L::SECOND : 0u, mine4 = gates4 + 128 * half;   // gates of this half's tokens
      Pair<M> so[HS];   // the other half of the state
#pragma unroll
      for (int s = 0; s < HS; ++s) so[s] = load_op<M>(hand + (HS * (1 - half) + s) * 2048);
      float o_unit = 1.f, k_inv = 1.f, y_inv = 1.f;
      if constexpr (HALF_E) k_inv = lds_read<float>(gates + 772);
      if constexpr (HALF_E) o_unit = lds_read<float>(units + 4 * i16 + (half ? 0 : 64));
      f32x4 x[2], xo[2], y[2], z[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) x[m] = xo[m] = y[m] = zero;
#pragma unroll
      for (int s = 0; s < HS; ++s)
#pragma unroll
        for (int m = 0; m < 2; ++m) x[m] = mma(kf[s][m], sp[s], x[m]);
      f32x4 since[2], other[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        since[m] = lds_read<f32x4>(mine4 + 64 * m);
        other[m] = lds_read<f32x4>(mine4 + (BACK ? 256 : 512) + 64 * m);
      }
      Opnd<E, 1> vf[2];   // columns of v of this half's tokens, or of dO of all
      if constexpr (BACK) {
        vf[0] = at_v.column(second, mine, 0);
        vf[1] = at_v.column(second, mine, 1);
      } else vf[0] = at_v.column(second + half * 4 * Tile<E, 64>::OCTET, mine, 0);
      Pair<M> tf[6];
      if constexpr (BACK) {   // P^T: its first four operands are the first half's rows, the others the second's
#pragma unroll
        for (int i = 0; i < 4; ++i) tf[i] = load_op<M>(ops + (half ? 4 + (i & 1) : i) * REC_OP);
      }
#pragma unroll
      for (int s = 0; s < HS; ++s)
#pragma unroll
        for (int m = 0; m < 2; ++m) xo[m] = mma(ko[s][m], so[s], xo[m]);
      if constexpr (BACK) {
        Opnd<M, 1> dof[2];
        if constexpr (COPIES) {   // dO as halves: one operand, times a power of two
          f32x4 d[4];
#pragma unroll
          for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) d[m][r] = (float)vf[m >> 1].t[0][4 * (m & 1) + r];
          const float unit = column_unit<M>(d);
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) dof[s].t[0][e] = (M)(d[2 * s + (e >> 2)][e & 3] * unit);
          y_inv = inverse_unit<M>(unit);
        } else {
          dof[0].t[0] = vf[0].t[0];
          dof[1].t[0] = vf[1].t[0];
        }
        if constexpr (HALF_E) y_inv *= k_inv * lds_read<float>(gates + 776);   // P^T has the units of keys and queries in it
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          if (half) y[m] = mma(tf[m], dof[1], y[m]);
          else y[m] = mma(tf[2 * m + 1], dof[1], mma(tf[2 * m], dof[0], y[m]));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 6; ++i) tf[i] = load_op<M>(ops + (BACK ? REC_TRIANGLE : 0) + i * REC_OP);   // T, or T^T
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const f32x4 ks = HALF_E ? (x[m] * inverse_unit<M>(s_unit) + xo[m] * inverse_unit<M>(o_unit)) * k_inv : x[m] + xo[m];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if constexpr (BACK) z[m][r] = a.scale * y_inv * y[m][r] + other[m][r] * ks[r];
          else z[m][r] = other[m][r] * ((float)vf[0].t[0][4 * m + r] - since[m][r] * ks[r]);
        }
      }
      {
        const float unit = column_unit<M>(z);
        Pair<M> zp[1];
        pairs_of<M>(zp, z, unit);
        write_op<M>(hand_z + half * 2048, zp[0]);
        if (HALF_E && lane < 16) lds_write(units + L::UNITS_Z + 64 * half + 4 * lane, unit);
      }
      __builtin_amdgcn_sched_barrier(0);
      Opnd<M, 1> kc[HT][2];   // columns of the keys, this half's rows of the state
#pragma unroll
      for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s) kc[i][s] = at.state_column(own, i, s);
      f32x4 factor[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        factor[m] = lds_read<f32x4>(gates4 + (BACK ? 512 : 256) + 64 * m);
        if constexpr (BACK) factor[m] *= -lds_read<f32x4>(gates4 + 64 * m);
      }
      const float whole = lds_read<float>(gates + 768);
      middle(n);
      Pair<M> zp[2];
      float zi[2] = {1.f, 1.f};
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        zp[s] = load_op<M>(hand_z + s * 2048);
        if constexpr (HALF_E) zi[s] = inverse_unit<M>(lds_read<float>(units + L::UNITS_Z + 64 * s + 4 * i16));
      }
      f32x4 add[HT];
      if constexpr (BACK)
#pragma unroll
        for (int i = 0; i < HT; ++i) add[i] = lds_read<f32x4>(hand_add + (HT * half + i) * 1024);
      at.move_state_places(AHEAD ? ((n & 1) ? (unsigned)-L::FIRST : (unsigned)L::FIRST) : 0u);
      f32x4 u[4], uo[4], next[4];   // uo: half's other tokens, which have a unit of their own
#pragma unroll
      for (int m = 0; m < 4; ++m) u[m] = uo[m] = zero;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int m = 0; m < 4; ++m)
          if (BACK ? s >= m / 2 : s <= m / 2) {
            const Pair<M>& t = tf[BACK ? upper_op(m, s) : lower_op(m, s)];
            if (HALF_E && s == 1) uo[m] = mma(t, zp[s], uo[m]);
            else u[m] = mma(t, zp[s], u[m]);
          }
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        if constexpr (HALF_E) u[m] = u[m] * zi[0] + uo[m] * zi[1];
        next[m] = u[m] * factor[m];
      }
      Pair<M> np[2];
      const float n_unit = column_unit<M>(next), n_inv = inverse_unit<M>(n_unit);
      pairs_of<M>(np, next, n_unit);
      if (AHEAD) load_keys();   // (behind the last chunk nothing is there, and nothing takes them)
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (HALF_E) {
        f32x4 p[HT];
#pragma unroll
        for (int i = 0; i < HT; ++i) p[i] = zero;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < HT; ++i) p[i] = mma(kc[i][s], np[s], p[i]);
#pragma unroll
        for (int i = 0; i < HT; ++i) {
          S[i] = S[i] * whole + p[i] * (n_inv * k_inv);
          if constexpr (BACK) S[i] += add[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < HT; ++i) S[i] = BACK ? S[i] * whole + add[i] : S[i] * whole;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < HT; ++i) S[i] = mma(kc[i][s], np[s], S[i]);
      }
      if (n + 1 < chunks) publish_state();
      end_chunk(n);
      if (!AHEAD && n + 1 < chunks) load_keys();
    }
    float* last = RESULTS ? a.ht : BACK ? a.dh0 : nullptr;
    if (last && live)
#pragma unroll
      for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at_row = state_row(HT * half + i, g, r);
          if (at_row < a.dk) last[((int64_t)doc * a.nv + h) * states + (int64_t)at_row * a.dv + col] = S[i][r];
        }
    return;
  }

  __syncthreads();
  if (LOADERS && loads) {
    for (int n = 0; n < chunks; ++n, c += step) {
      begin_chunk(n);
      middle(n);
      end_chunk(n);
    }
    return;
  }
  // Tokens, and rows of the state, in 16s: a helper has its part of HELPERS of them.
  auto help = [&](auto part) {
    constexpr int MT = 4 / HELPERS, M0 = part.value * MT;
    if constexpr (RESULTS) {
      constexpr int UT = M0 + MT;   // of u: what P's rows are not zero for
      TileOps<M, DK> at;
      at.state_places(smem + L::Q, lane);
      for (int n = 0; n < chunks; ++n, c += step) {
        const unsigned gates = smem + (AHEAD ? (unsigned)(n & 1) * L::FIRST : 0u) + L::R, ops = gates + REC_GATES + 16 * lane;
        begin_chunk(n);
        Pair<M> sf[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) sf[s] = load_op<M>(hand + s * 2048);
        f32x4 back_s[2];   // half: of the rows' columns, of either half of the state
        if constexpr (HALF_E) {
          back_s[0] = lds_read<f32x4>(units + 16 * g);
          back_s[1] = lds_read<f32x4>(units + 64 + 16 * g);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            back_s[0][r] = inverse_unit<M>(back_s[0][r]);
            back_s[1][r] = inverse_unit<M>(back_s[1][r]);
          }
        }
        float q_inv = 1.f, p_inv = 1.f;
        if constexpr (HALF_E) {
          q_inv = lds_read<float>(gates + 776);
          p_inv = q_inv * lds_read<float>(gates + 772);
        }
        f32x4 o[MT], oo[MT];   // transposed: rows are columns of the state, a lane has the token lane % 16
        float zi[2];         // half: the inverse units of Z
        Pair<M> pf[6], tf[6], zp[2];   // those that these tiles need
#pragma unroll
        for (int m = 0; m < MT; ++m) o[m] = oo[m] = zero;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            if (HALF_E && s >= HS) oo[m] = mma(sf[s], at.state_row(0, M0 + m, s), oo[m]);
            else o[m] = mma(sf[s], at.state_row(0, M0 + m, s), o[m]);
          }
        if constexpr (ALL_AHEAD) at.move_state_places((n & 1) ? (unsigned)-L::SECOND : (unsigned)L::SECOND);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const float since = lds_read<float>(gates + 4 * (16 * (M0 + m) + i16));
          if constexpr (HALF_E) o[m] = (o[m] * back_s[0] + oo[m] * back_s[1]) * (since * q_inv);
          else o[m] *= since;
        }
#pragma unroll
        for (int i = 0; i < 6; ++i) {
          tf[i] = load_op<M>(ops + i * REC_OP);
          pf[i] = load_op<M>(ops + REC_TRIANGLE + i * REC_OP);
        }
        middle(n);
        zp[0] = load_op<M>(hand_z);
        zp[1] = load_op<M>(hand_z + 2048);
        if constexpr (HALF_E)
#pragma unroll
          for (int s = 0; s < 2; ++s) zi[s] = inverse_unit<M>(lds_read<float>(units + L::UNITS_Z + 4 * i16 + 64 * s));
        f32x4 u[UT], uo[UT], p[MT], back_u = zero;
#pragma unroll
        for (int m = 0; m < UT; ++m) u[m] = uo[m] = zero;
#pragma unroll
        for (int s = 0; s < UT / 2; ++s)
#pragma unroll
          for (int m = 0; m < UT; ++m)
            if (s <= m / 2) {
              if (HALF_E && s == 1) uo[m] = mma(tf[lower_op(m, s)], zp[s], uo[m]);
              else u[m] = mma(tf[lower_op(m, s)], zp[s], u[m]);
            }
        if constexpr (HALF_E)
#pragma unroll
          for (int m = 0; m < UT; ++m) u[m] = u[m] * zi[0] + uo[m] * zi[1];
        Pair<M> up[UT / 2];
        const float unit = column_unit<M>(u), inv = inverse_unit<M>(unit);
        pairs_of<M>(up, u, unit);
        if constexpr (HALF_E) {
#pragma unroll
          for (int r = 0; r < 4; ++r) back_u[r] = __shfl(inv, 4 * g + r, 64);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) p[m] = HALF_E ? zero : o[m];
#pragma unroll
        for (int s = 0; s < UT / 2; ++s)
#pragma unroll
          for (int m = 0; m < MT; ++m)
            if (s <= (M0 + m) / 2) p[m] = mma(up[s], pf[lower_op(M0 + m, s)], p[m]);
        E* oh = (E*)a.o + h * a.dv + w0 + 4 * g;
        if (w0 + 4 * g < a.dv)
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const int t = DELTA_C * c + 16 * (M0 + m) + i16;
            if constexpr (HALF_E) p[m] = p[m] * (back_u * p_inv) + o[m];
            if (t < count) {
              typedef E quad_t __attribute__((ext_vector_type(4)));
              quad_t w;
#pragma unroll
              for (int r = 0; r < 4; ++r) w[r] = from_f<E>(fp32_value(p[m][r] * a.scale));
              *reinterpret_cast<quad_t*>(oh + (first + t) * a.ldo) = w;
            }
          }
        end_chunk(n);
      }
    } else {
      constexpr int IT = RT / HELPERS, I0 = part.value * IT;
      TileOps<M, DK> at;
      at.state_places(smem + L::Q, lane);
      const TileOps<E, 64> at_v(smem + L::V, lane);
      for (int n = 0; n < chunks; ++n, c += step) {
        const unsigned gates = smem + (AHEAD ? (unsigned)(n & 1) * L::FIRST : 0u) + L::R, gates4 = gates + 16 * g, ops = gates + REC_GATES + 16 * lane;
        const int64_t rec = (int64_t)(chunk0 + c) * a.nv + h;
        begin_chunk(n);
        // The state, as its pairs are, for the gradients' products.  Half: read transposed, so that a lane has four columns of a row, and stored in the
        // other phase: as a lane's rows of one column, 32 stores of 4 bytes, this wave kept the chain waiting for 2000 cycles a chunk.
        float* to = (BACK ? a.dstates : a.states) + rec * DK * a.dvp;
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        union Quad { s16x4 w; f16 v[4]; } sq[HALF_E ? IT : 1][2];
        f32x4 inv[2];
        if constexpr (HALF_E) {
          const unsigned across = hand - 16 * lane + 256 * ((i16 & 3) >> 1) + 64 * g + 16 * (i16 >> 2) + 8 * (i16 & 1);
#pragma unroll
          for (int i = 0; i < IT; ++i)
#pragma unroll
            for (int p = 0; p < 2; ++p)
              sq[i][p].w = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(across + ((I0 + i) >> 1) * 2048 + p * 1024 + ((I0 + i) & 1) * 512));
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            inv[p] = lds_read<f32x4>(units + 64 * p + 16 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) inv[p][r] = inverse_unit<M>(inv[p][r]);
          }
        } else if (col < a.dvp) {
#pragma unroll
          for (int s = I0 / 2; s < (I0 + IT) / 2; ++s) {
            const Pair<M> sf = load_op<M>(hand + s * 2048);
#pragma unroll
            for (int e = 0; e < 8; ++e) to[(32 * s + 8 * g + e) * a.dvp + col] = sf.t[0][e];
          }
        }
        if constexpr (BACK) {   // scale Q^T (exp(G) dO)
          const unsigned second = ALL_AHEAD ? (unsigned)(n & 1) * L::SECOND : 0u;
          Opnd<E, 1> vf[2];
          vf[0] = at_v.column(second, mine, 0);
          vf[1] = at_v.column(second, mine, 1);
          f32x4 d[4], add[IT];
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const f32x4 since = lds_read<f32x4>(gates4 + 64 * m);
#pragma unroll
            for (int r = 0; r < 4; ++r) d[m][r] = a.scale * since[r] * (float)vf[m >> 1].t[0][4 * (m & 1) + r];
          }
          Pair<M> dp[2];
          const float unit = column_unit<M>(d), back = inverse_unit<M>(unit);
          pairs_of<M>(dp, d, unit);
#pragma unroll
          for (int i = 0; i < IT; ++i) add[i] = zero;
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < IT; ++i) add[i] = mma(at.state_column(0, I0 + i, s), dp[s], add[i]);
          if constexpr (ALL_AHEAD) at.move_state_places((n & 1) ? (unsigned)-L::SECOND : (unsigned)L::SECOND);
#pragma unroll
          for (int i = 0; i < IT; ++i) lds_write(hand_add + (I0 + i) * 1024, HALF_E ? add[i] * (back * lds_read<float>(gates + 776)) : add[i]);
        }
        Pair<M> tf[6], zp[2];
#pragma unroll
        for (int i = 0; i < 6; ++i) tf[i] = load_op<M>(ops + (BACK ? REC_TRIANGLE : 0) + i * REC_OP);
        middle(n);
        if constexpr (HALF_E) {
          if (w0 < a.dvp)
#pragma unroll
            for (int i = 0; i < IT; ++i) {
              f32x4 x;
#pragma unroll
              for (int r = 0; r < 4; ++r) x[r] = ((float)sq[i][0].v[r] + (float)sq[i][1].v[r]) * inv[I0 + i >= HT][r];
              *reinterpret_cast<f32x4*>(to + (16 * (I0 + i) + i16) * a.dvp + w0 + 4 * g) = x;
            }
        }
        f32x4 u[MT], uo[MT], back_z[2];   // transposed: rows are columns of the state
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          zp[s] = load_op<M>(hand_z + s * 2048);
          if constexpr (HALF_E) {
            back_z[s] = lds_read<f32x4>(units + L::UNITS_Z + 64 * s + 16 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) back_z[s][r] = inverse_unit<M>(back_z[s][r]);
          }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) u[m] = uo[m] = zero;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int m = 0; m < MT; ++m)
            if (BACK ? s >= (M0 + m) / 2 : s <= (M0 + m) / 2) {
              const Pair<M>& t = tf[BACK ? upper_op(M0 + m, s) : lower_op(M0 + m, s)];
              if (HALF_E && s == 1) uo[m] = mma(zp[s], t, uo[m]);
              else u[m] = mma(zp[s], t, u[m]);
            }
        float* to_u = (BACK ? a.y : a.u) + rec * DELTA_C * a.dvp + i16 * a.dvp + w0 + 4 * g;
        if (w0 + 4 * g < a.dvp)
#pragma unroll
          for (int m = 0; m < MT; ++m) *reinterpret_cast<f32x4*>(to_u + 16 * (M0 + m) * a.dvp) = HALF_E ? u[m] * back_z[0] + uo[m] * back_z[1] : u[m];
        end_chunk(n);
      }
    }
  };
  if (wave < 3 * NW) help(Int<BACK ? 0 : 1>());
  else help(Int<BACK ? 1 : 0>());   // the smaller one
}

// Block of the grid -> document and head, and columns: the blocks that share keys and matrices lie eight apart, on one XCD.
struct WalkBlock { int doc, h, c0; bool in; };
__device__ __forceinline__ WalkBlock walk_block(const DeltaRule& a, int block, int slices, int width) {
  const int j = block / 8, pair = j / slices * 8 + block % 8;
  return WalkBlock{pair / a.nv, pair % a.nv, j % slices * width, pair < a.ndocs * a.nv};
}
template <typename E, typename M, int DK, int NW> __global__ __launch_bounds__(walk_threads(NW), 1) void delta_walk_kernel(DeltaRule a, int slices) {
  __shared__ __align__(16) char smem[WalkLds<E, M, DK, NW, WALK_RESULTS>::BYTES];
  const WalkBlock b = walk_block(a, blockIdx.x, slices, 16 * NW);
  if (b.in) delta_walk<E, M, DK, NW, WALK_RESULTS>(smem, a, b.doc, b.h, b.c0);
}
// Both walks of the backward: they need nothing of one another.
template <typename E, int DK, int NW> __global__ __launch_bounds__(walk_threads(NW), 1) void delta_walks_kernel(DeltaRule a, int slices, int blocks) {
  typedef typename WalkOf<E>::type M;
  constexpr int LS = WalkLds<E, M, DK, NW, WALK_STATES>::BYTES, LG = WalkLds<E, M, DK, NW, WALK_GRADIENTS>::BYTES;
  __shared__ __align__(16) char smem[LS > LG ? LS : LG];
  const bool back = (int)blockIdx.x < blocks;
  const WalkBlock b = walk_block(a, back ? (int)blockIdx.x : (int)blockIdx.x - blocks, slices, 16 * NW);
  if (!b.in) return;
  if (back) delta_walk<E, M, DK, NW, WALK_GRADIENTS>(smem, a, b.doc, b.h, b.c0);
  else delta_walk<E, M, DK, NW, WALK_STATES>(smem, a, b.doc, b.h, b.c0);
}

// ------------------------------------------------------------------------------------------ gradients of a chunk
// What the products take their operands in: half as bf16 pairs, whose exponent holds whatever a gradient may be (a half is exactly such a pair).
template <typename E> struct GradOf { typedef bf16 type; };
template <> struct GradOf<float> { typedef float type; };
template <typename E> constexpr int GRAD_IN = __is_same(E, f16) ? 2 : 1;
template <typename E> __device__ __forceinline__ Opnd<typename GradOf<E>::type, GRAD_IN<E>> grad_in(const Opnd<E, 1>& x) {
  if constexpr (__is_same(E, f16)) {
    Opnd<bf16, 2> o;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = (float)x.t[0][e];
      o.t[0][e] = (bf16)v;
      o.t[1][e] = (bf16)(v - (float)o.t[0][e]);
    }
    return o;
  } else return x;
}

template <typename M> constexpr int GRAD_TERMS = sizeof(M) == 2 ? 3 : 1;
template <typename M> using GradOpnd = Opnd<M, GRAD_TERMS<M>>;
template <typename M> __device__ __forceinline__ void write_terms(unsigned lds_of_lane, const GradOpnd<M>& x) {
  union { GradOpnd<M> v; f32x4 h[sizeof(x) / 16]; } u;
  u.v = x;
#pragma unroll
  for (int p = 0; p < (int)sizeof(x) / 16; ++p) lds_write(lds_of_lane + p * 1024, u.h[p]);
}
template <typename M> __device__ __forceinline__ GradOpnd<M> load_terms(unsigned lds_of_lane) {
  union { GradOpnd<M> v; f32x4 h[sizeof(GradOpnd<M>) / 16]; } u;
#pragma unroll
  for (int p = 0; p < (int)sizeof(u) / 16; ++p) u.h[p] = lds_read<f32x4>(lds_of_lane + p * 1024);
  return u.v;
}

// A workgroup per chunk and key head; the value heads of the key head one after the other, their dq and dk in the same registers.  A wave has 16 of the
// head's columns of dq and dk, for all tokens: results are transposed (rows are columns of the head, a lane has a token), so that a
// state's rows are read by one wave only and a token's factors are a lane's own.  The matrices of tokens by tokens are shared out by tiles: wave
// w has the row tile w % 4, and of its column tiles those of its parity where there are eight waves.  Columns of the value head come in blocks of 64.
// A workgroup fills a CU (157 KB of LDS, 242 registers), so what it loads is asked for ahead, states 32 columns, u and y 64, and the first of them before its
// row of the table is there.  4096 tokens of 16 heads of 128 in bf16: 120 us in 4.3 rounds of 256 workgroups, 278 MB read at 2.3 TB/s (214 of them states, u and
// y), the matrix cores busy in 0.15 of the cycles; a workgroup's phases follow one another: of 45000 cycles alone 12700 until the first loads are there, 10800 the
// products with states, 8600 the matrices of tokens and the sums over them, 7300 the products with these, and fewer registers would spill (128, two
// workgroups a CU: 245 us).
constexpr int grad_waves(int DK) { return DK / 16; }
template <typename E, int DK, bool SHARED> __global__ __launch_bounds__(64 * grad_waves(DK), 1) void delta_grad_kernel(DeltaRule a) {
  typedef typename GradOf<E>::type M;
  typedef Opnd<M, GRAD_IN<E>> In;
  typedef Tile<E, DK> TL;
  typedef Tile<E, 64> VL;
  constexpr int W = grad_waves(DK), PARTS = W / 4, TILE = TL::bytes(DELTA_C), KS = DK / 32, OP = sizeof(GradOpnd<M>) * 64, OPS = 8 * OP;   // OPS: 64 tokens by 64 columns as operands
  struct Sums { float m[2][64][TRI_LD], dots[W][3][64], cols[4][64], rows[PARTS][2][64], whole[W]; };   // over the columns' blocks, when these are through
  constexpr int BLOCKS = VL::bytes(DELTA_C) + 2 * OPS, STAGE = sizeof(Sums) > BLOCKS ? sizeof(Sums) : BLOCKS;
  __shared__ __align__(16) char smem_raw[2 * TILE + STAGE + 20 * REC_OP];
  __shared__ double G[64];
  __shared__ float gate[4][64], yvs[2][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, i16 = lane & 15;
  const ChunkRow c = chunk_row(a, blockIdx.x);
  const int kv = blockIdx.y, group = SHARED ? a.nv / a.nk : 1, tile = wave & 3, part = wave >> 2;
  const unsigned smem = lds_address(smem_raw), stage = 2 * TILE;
  typedef E quad_t __attribute__((ext_vector_type(4)));
  const int my_t = 16 * tile + i16;         // the token whose rows of U and Y this lane brings, of 64 columns or, as one of eight waves, of 32
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 sx[2], sy[2];                       // rows of S and dS, 32 columns ahead
  f32x4 u[2 / PARTS][2], y[2 / PARTS][2];   // rows of U, Y and v, 64 columns ahead
  quad_t v[2 / PARTS][2];
  float my_gate = 0.f;
  double my_G = 0.0;
  // Through descriptors: an address is a register, and what lies behind a matrix, or in columns past its width, reads as zeros.
  const unsigned my_state = (unsigned)((16 * wave + i16) * a.dvp + 4 * g) * 4, my_row = (unsigned)(my_t * a.dvp + 4 * g) * 4;
  auto matrix = [&](const float* p, int rows) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p), 0, rows * a.dvp * 4, 0x00020000); };
  auto quad_at = [&](const __amdgpu_buffer_rsrc_t& m, unsigned lane_at, int col) {
    union { u32x4 w; f32x4 v; } x;
    x.w = __builtin_amdgcn_raw_buffer_load_b128(m, lane_at + (col < a.dvp ? 4u * col : 0x80000000u), 0, 0);
    return x.v;
  };
  auto load_states = [&](int64_t rec, int col0) {
    const __amdgpu_buffer_rsrc_t S = matrix(a.states + rec * DK * a.dvp, DK), dS = matrix(a.dstates + rec * DK * a.dvp, DK);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      sx[p] = quad_at(S, my_state, col0 + 16 * p);
      sy[p] = quad_at(dS, my_state, col0 + 16 * p);
    }
  };
  auto load_rows = [&](int64_t rec, int b0) {
    const __amdgpu_buffer_rsrc_t U = matrix(a.u + rec * DELTA_C * a.dvp, DELTA_C), Y = matrix(a.y + rec * DELTA_C * a.dvp, DELTA_C);
#pragma unroll
    for (int s = 0; s < 2 / PARTS; ++s)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        u[s][p] = quad_at(U, my_row, b0 + 32 * (s + part) + 16 * p);
        y[s][p] = quad_at(Y, my_row, b0 + 32 * (s + part) + 16 * p);
      }
  };
  auto load_v = [&](int h, int b0) {
    const __amdgpu_buffer_rsrc_t vs = __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>((const E*)a.v + (int64_t)c.first * a.ldv + h * a.dv), 0,
                                                                        (int)(((c.count - 1) * a.ldv + a.dv) * sizeof(E)), 0x00020000);
#pragma unroll
    for (int s = 0; s < 2 / PARTS; ++s)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int col = b0 + 32 * (s + part) + 16 * p + 4 * g;
        const unsigned at_v = col < a.dv ? (unsigned)(my_t * (int)a.ldv + col) * (unsigned)sizeof(E) : 0x80000000u;
        if constexpr (sizeof(E) == 4) {
          union { u32x4 w; quad_t v; } x;
          x.w = __builtin_amdgcn_raw_buffer_load_b128(vs, at_v, 0, 0);
          v[s][p] = x.v;
        } else {
          union { u32x2 w; quad_t v; } x;
          x.w = __builtin_amdgcn_raw_buffer_load_b64(vs, at_v, 0, 0);
          v[s][p] = x.v;
        }
      }
  };
  auto load_head = [&](int64_t rec) {
    const char* from = a.records + rec * REC_BWD;
    if (wave < 4) my_gate = reinterpret_cast<const float*>(from)[64 * wave + lane];
    if (wave == 0) my_G = reinterpret_cast<const double*>(from + REC_G)[lane];
    load_rows(rec, 0);
    load_states(rec, 0);
  };
  load_head((int64_t)blockIdx.x * a.nv + kv * group);   // while the chunk's row of the table is still under way
  __builtin_amdgcn_sched_barrier(0);
  if (c.count <= 0) return;
  const int end = c.first + c.count;
  const bool my_in = my_t < c.count;
  auto fetch_do = [&](int h, int b0) {
    const TileLoad<E, 64, DELTA_C, W> load(a.ldo, lane, min(a.dv - b0, 64));
    tile_ahead(load, smem + stage, (const E*)a.dout + h * a.dv + b0, c.first, end, wave);
  };
  load_v(kv * group, 0);
  fetch_do(kv * group, 0);
  {
    const TileLoad<E, DK, DELTA_C, W> load_k(a.ldk, lane, a.dk), load_q(a.ldq, lane, a.dk);
    tile_ahead(load_k, smem, (const E*)a.k + kv * a.dk, c.first, end, wave);
    tile_ahead(load_q, smem + TILE, (const E*)a.q + kv * a.dk, c.first, end, wave);
  }
  const TileOps<E, DK> at(smem, lane);
  const TileOps<E, 64> at_do(smem + stage, lane);
  const unsigned n_ops = smem + stage + VL::bytes(DELTA_C) + 16 * lane, y_ops = n_ops + OPS;
  Sums& sums = *reinterpret_cast<Sums*>(smem_raw + stage);
  float *Mm = sums.m[0][0], *H = sums.m[1][0];
  const unsigned m_ops = smem + stage + STAGE + 16 * lane;
  f32x4 dq[4], dk[4];
#pragma unroll
  for (int n = 0; n < 4; ++n) dq[n] = dk[n] = zero;
  for (int hg = 0; hg < group; ++hg) {
    const int h = kv * group + hg;
    const int64_t rec = (int64_t)blockIdx.x * a.nv + h;
    if (SHARED && hg > 0) {
      __syncthreads();   // the head before is done with the LDS
      load_head(rec);
      load_v(h, 0);
      fetch_do(h, 0);
    }
    if (wave < 4) gate[wave][lane] = my_gate;
    if (wave == 0) G[lane] = my_G;
    f32x4 qi[4], ks[4], kn[4], dp[4 / PARTS], da[4 / PARTS];
#pragma unroll
    for (int n = 0; n < 4; ++n) qi[n] = ks[n] = kn[n] = zero;
#pragma unroll
    for (int n = 0; n < 4 / PARTS; ++n) dp[n] = da[n] = zero;
    float sds = 0.f, yv = 0.f;
    for (int b0 = 0; b0 < a.dv; b0 += 64) {
      __syncthreads();   // the block before has been read; the gates are there
      if (b0 > 0) fetch_do(h, b0);
      const float beta = gate[2][my_t];
#pragma unroll
      for (int s = 0; s < 2 / PARTS; ++s) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const int col = b0 + 32 * (s + part) + 16 * p + 4 * g;
          quad_t w;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            yv = fmaf(y[s][p][e], (float)v[s][p][e], yv);
            w[e] = from_f<E>(fp32_value(beta * y[s][p][e]));
          }
          if (my_in && col < a.dv) *reinterpret_cast<quad_t*>((E*)a.dval + (int64_t)(c.first + my_t) * a.lddv + h * a.dv + col) = w;
        }
        write_terms<M>(n_ops + (2 * tile + s + part) * OP, terms_of<M, GRAD_TERMS<M>>(u[s][0], u[s][1]));
        write_terms<M>(y_ops + (2 * tile + s + part) * OP, terms_of<M, GRAD_TERMS<M>>(y[s][0], y[s][1]));
      }
      tile_wait();
      __syncthreads();
      __builtin_amdgcn_sched_barrier(0);
      load_rows(rec, b0 + 64);   // (zeros behind the last)
      load_v(h, b0 + 64);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int e = 0; e < 4; ++e) sds = fmaf(sx[p][e], sy[p][e], sds);
        const GradOpnd<M> sp = terms_of<M, GRAD_TERMS<M>>(sx[0], sx[1]), dsp = terms_of<M, GRAD_TERMS<M>>(sy[0], sy[1]);
        __builtin_amdgcn_sched_barrier(0);
        load_states(rec, b0 + 32 * (s + 1));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const In d = grad_in<E>(at_do.row(0, m, s));
          const GradOpnd<M> un = load_terms<M>(n_ops + (2 * m + s) * OP), yn = load_terms<M>(y_ops + (2 * m + s) * OP);
          qi[m] = mma(sp, d, qi[m]);
          ks[m] = mma(sp, yn, ks[m]);
          kn[m] = mma(dsp, un, kn[m]);
        }
        const In d_i = grad_in<E>(at_do.row(0, tile, s));
        const GradOpnd<M> y_i = load_terms<M>(y_ops + (2 * tile + s) * OP);
#pragma unroll
        for (int n = 0; n < 4 / PARTS; ++n)
          if (PARTS * n + part <= tile) {
            const GradOpnd<M> u_j = load_terms<M>(n_ops + (2 * (PARTS * n + part) + s) * OP);
            dp[n] = mma(d_i, u_j, dp[n]);
            da[n] = mma(y_i, u_j, da[n]);
          }
      }
    }
    f32x4 kk[4 / PARTS], qk[4 / PARTS];
#pragma unroll
    for (int n = 0; n < 4 / PARTS; ++n) kk[n] = qk[n] = zero;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const Opnd<E, 1> k_i = at.row(0, tile, s), q_i = at.row(TILE, tile, s);
#pragma unroll
      for (int n = 0; n < 4 / PARTS; ++n)
        if (PARTS * n + part <= tile) {
          const Opnd<E, 1> k_j = at.row(0, PARTS * n + part, s);
          kk[n] = mma(k_i, k_j, kk[n]);
          qk[n] = mma(q_i, k_j, qk[n]);
        }
    }
    __syncthreads();   // the sums lie over the blocks
    // the states' shares, and their products with q and k
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const float since = gate[0][16 * m + i16], until = gate[1][16 * m + i16], beta = gate[2][16 * m + i16];
      float dot[3] = {0.f, 0.f, 0.f};
      const f32x4 k4 = at.quad(0, m, wave), q4 = at.quad(TILE, m, wave);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float q_state = a.scale * since * qi[m][r], k_state = -since * ks[m][r], k_next = until * kn[m][r];
        dot[0] = fmaf(q4[r], q_state, dot[0]);
        dot[1] = fmaf(k4[r], k_state, dot[1]);
        dot[2] = fmaf(k4[r], k_next, dot[2]);
        dq[m][r] += q_state;
        dk[m][r] += fmaf(beta, k_state, k_next);
      }
#pragma unroll
      for (int x = 0; x < 3; ++x) {
        dot[x] = rows_sum(dot[x]);
        if (lane < 16) sums.dots[wave][x][16 * m + lane] = dot[x];
      }
    }
    sds = wave_sum(sds);
    yv = rows_sum(yv);
    if (lane == 0) sums.whole[wave] = sds;
    if (lane < 16) yvs[part][16 * tile + lane] = yv;
    // M and H, and the sums by rows and by columns that the decays and beta get
    {
      float by_row[4] = {0.f, 0.f, 0.f, 0.f}, by_beta[4] = {0.f, 0.f, 0.f, 0.f};
      double gi[4];
      float bi[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        gi[r] = G[16 * tile + 4 * g + r];
        bi[r] = gate[2][16 * tile + 4 * g + r];
      }
#pragma unroll
      for (int n = 0; n < 4 / PARTS; ++n) {
        const int nt = PARTS * n + part, j = 16 * nt + i16;
        const double gj = G[j];
        float by_col = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int i = 16 * tile + 4 * g + r;
          const float dec = j <= i && nt <= tile ? decay(gi[r], gj) : 0.f;
          const float m = a.scale * dec * dp[n][r], hb = j < i ? -dec * da[n][r] : 0.f;
          Mm[i * TRI_LD + j] = m;
          H[i * TRI_LD + j] = bi[r] * hb;
          const float e = fmaf(m, qk[n][r], bi[r] * hb * kk[n][r]);
          by_row[r] += e;
          by_beta[r] = fmaf(hb, kk[n][r], by_beta[r]);
          by_col += e;
        }
        by_col = rows_sum(by_col);
        if (lane < 16) sums.cols[tile][j] = by_col;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        by_row[r] = columns_sum(by_row[r]);
        by_beta[r] = columns_sum(by_beta[r]);
        if (i16 == 0) {
          sums.rows[part][0][16 * tile + 4 * g + r] = by_row[r];
          sums.rows[part][1][16 * tile + 4 * g + r] = by_beta[r];
        }
      }
    }
    __syncthreads();
    if (wave == W - 1) {
      double d = 0.0, kn_sum = 0.0, sds_sum = 0.0;
      float kst = 0.f, knx = 0.f, qst = 0.f, db = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) d -= sums.cols[w][lane];
#pragma unroll
      for (int w = 0; w < PARTS; ++w) {
        d += sums.rows[w][0][lane];
        db += sums.rows[w][1][lane] + yvs[w][lane];
      }
#pragma unroll
      for (int w = 0; w < W; ++w) {
        qst += sums.dots[w][0][lane];
        kst += sums.dots[w][1][lane];
        knx += sums.dots[w][2][lane];
        sds_sum += sums.whole[w];
      }
      kn_sum = knx;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) kn_sum += __shfl_xor(kn_sum, o, 64);
      d += (double)qst + (double)gate[2][lane] * kst - knx;
      if (lane == 63) d += kn_sum + (double)gate[3][0] * sds_sum;
      // from each token to the end
      const double upto = running_sum(d, lane), all = __shfl(upto, 63, 64);
      if (lane < c.count) {
        const int64_t t = (int64_t)(c.first + lane) * a.nv + h;
        a.dg[t] = (float)(all - upto + d);
        a.dbeta[t] = db + kst;
      }
    }
    // M, M^T and H + H^T as operands, shared out over the waves: eight of the last, six of each of the others
    for (int k = wave; k < 20; k += W) {
      const int j = k < 8 ? k : k < 14 ? k - 8 : k - 14, m = k < 8 ? j >> 1 : k < 14 ? (j < 2 ? j : 1 + j / 2) : (j < 4 ? j >> 1 : j - 2),
                s = k < 8 ? j & 1 : k < 14 ? (j < 2 ? 0 : j & 1) : (j < 4 ? j & 1 : 1);
      const int from = 32 * s + 4 * g, mine = 16 * m + i16;
      const float* mat = k < 8 ? H : Mm;
      f32x4 x[2] = {zero, zero};
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (k < 14) x[p] = *reinterpret_cast<const f32x4*>(mat + mine * TRI_LD + from + 16 * p);
        if (k < 8 || k >= 14)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[p][e] += mat[(from + 16 * p + e) * TRI_LD + mine];
      }
      write_op<M>(m_ops + k * REC_OP, pair_of<M>(x[0], x[1]));
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const In k_col = grad_in<E>(at.column(0, wave, s)), q_col = grad_in<E>(at.column(TILE, wave, s));
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        dk[m] = mma(k_col, load_op<M>(m_ops + (2 * m + s) * REC_OP), dk[m]);
        if (s <= m / 2) dq[m] = mma(k_col, load_op<M>(m_ops + (8 + lower_op(m, s)) * REC_OP), dq[m]);
        if (s >= m / 2) dk[m] = mma(q_col, load_op<M>(m_ops + (14 + upper_op(m, s)) * REC_OP), dk[m]);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int col = 16 * wave + 4 * g, tok = 16 * m + i16;
    if (tok < c.count && col < a.dk) {
      quad_t x, y;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] = from_f<E>(fp32_value(dq[m][r]));
        y[r] = from_f<E>(fp32_value(dk[m][r]));
      }
      *reinterpret_cast<quad_t*>((E*)a.dq + (int64_t)(c.first + tok) * a.lddq + kv * a.dk + col) = x;
      *reinterpret_cast<quad_t*>((E*)a.dkey + (int64_t)(c.first + tok) * a.lddk + kv * a.dk + col) = y;
    }
  }
}

// ------------------------------------------------------------------------------------------ launches
template <typename E, typename M, int DK, int NW> hipError_t delta_walk_results(hipStream_t st, const DeltaRule& a) {
  const int slices = (int)cdiv(a.dv, 16 * NW), blocks = (int)(cdiv((int64_t)a.ndocs * a.nv, 8) * 8 * slices);
  hipLaunchKernelGGL((delta_walk_kernel<E, M, DK, NW>), dim3((unsigned)blocks), dim3(walk_threads(NW)), 0, st, a, slices);
  return hipGetLastError();
}
template <typename E, int DK, int NW> hipError_t delta_walks(hipStream_t st, const DeltaRule& a) {
  const int slices = (int)cdiv(a.dv, 16 * NW), blocks = (int)(cdiv((int64_t)a.ndocs * a.nv, 8) * 8 * slices);
  hipLaunchKernelGGL((delta_walks_kernel<E, DK, NW>), dim3((unsigned)(2 * blocks)), dim3(walk_threads(NW)), 0, st, a, slices, blocks);
  return hipGetLastError();
}
// Workgroups of 32 columns share what they bring into LDS; of 16 where 32 would leave CUs without one.  bf16, widths of 128, us of the walk with 16 and 32: 3
// documents of 4 heads (96 sets of 16 columns) 6.0 and 8.5, one of 32 heads (256) 177 and 229, 6 of 16 heads (768) 51.5 and 47, backward (1536) 145 and 110;
// half, 6 of 8 heads (576) 35.8 and 34.
inline bool walks_are_wide(const DeltaRule& a, int walks) { return (int64_t)a.ndocs * a.nv * cdiv(a.dv, 16) * walks >= 512; }
template <typename E, typename M, int DK> hipError_t delta_forward(hipStream_t st, const DeltaRule& a) {
  hipLaunchKernelGGL((delta_prep_kernel<E, M, DK, false>), dim3((unsigned)(a.nchunks + DELTA_FILL), (unsigned)a.nk), dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.ndocs == 0) return e;
  return walks_are_wide(a, 1) ? delta_walk_results<E, M, DK, 2>(st, a) : delta_walk_results<E, M, DK, 1>(st, a);
}
template <typename E, int DK> hipError_t delta_backward(hipStream_t st, const DeltaRule& a) {
  hipLaunchKernelGGL((delta_prep_kernel<E, typename WalkOf<E>::type, DK, true>), dim3((unsigned)(a.nchunks + DELTA_FILL), (unsigned)a.nk), dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.ndocs == 0) return e;
  e = walks_are_wide(a, 2) ? delta_walks<E, DK, 2>(st, a) : delta_walks<E, DK, 1>(st, a);
  if (e != hipSuccess || a.nchunks == 0) return e;
  const dim3 grid((unsigned)a.nchunks, (unsigned)a.nk);
  if (a.nv == a.nk) hipLaunchKernelGGL((delta_grad_kernel<E, DK, false>), grid, dim3(64 * grad_waves(DK)), 0, st, a);
  else hipLaunchKernelGGL((delta_grad_kernel<E, DK, true>), grid, dim3(64 * grad_waves(DK)), 0, st, a);
  return hipGetLastError();
}
template <typename E, int DK> hipError_t delta_run(hipStream_t st, const DeltaRule& a, bool backward) {
  if (backward) return delta_backward<E, DK>(st, a);
  // Rounded results need less than last states do.  bf16, widths of 128, the whole call: 4096 tokens in documents, 16 heads, 66 us and with last states 78; one
  // document of 8192, 32 heads over 16, 204 and 268.
  return a.ht ? delta_forward<E, typename WalkOf<E>::type, DK>(st, a) : delta_forward<E, E, DK>(st, a);
}
template <typename E> hipError_t delta_rule_of(hipStream_t st, const DeltaRule& a, bool backward) {
  return a.dk <= 64 ? delta_run<E, 64>(st, a, backward) : delta_run<E, 128>(st, a, backward);
}

}  // namespace
}  // namespace zs
