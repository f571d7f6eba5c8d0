// What the matrix-core kernels of attention inside packed documents share: tiles of rows in LDS, fragments of them, the products of an
// element type, and the blocks' ranges.
//
// All products are computed transposed (S^T = K Q^T, O^T = V^T P^T and so on) on 32 x 32 blocks: a lane then owns one query (or key), lane
// % 32, and its registers hold the block's rows 8 (r/4) + 4 (lane/32) + r%4, which is, converted to the type, the operand that the
// next product wants.  16-bit types: v_mfma_f32_32x32x16; fp32: v_mfma_f32_32x32x2, as many of them as it takes, on the same layout.
#pragma once
#include "attention_docs_rows.h"

namespace zs {
namespace {

constexpr float DOC_LOG2E = 1.4426950408889634f;
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ int acc_row(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// A type's 16 bytes along a row (vec), and 8 rows of a column (col8): of the rows 16 s + 4 (lane/32) + {0 .. 3, 8 .. 11}, in the order
// of the accumulators 8 s .. 8 s + 7.
template <typename E> struct Mat {
  typedef typename Vec<E>::type vec;
  typedef vec col8;
  static __device__ __forceinline__ f32x16 mma(vec a, vec b, f32x16 c) {
    if constexpr (sizeof(E) == 2 && __is_same(E, bf16)) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 rows(vec a, vec b, f32x16 c) { return mma(a, b, c); }
  static __device__ __forceinline__ f32x16 cols(col8 a, col8 b, f32x16 c) { return mma(a, b, c); }
  static __device__ __forceinline__ col8 pack(const f32x16& x, int s) {
    col8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (E)x[8 * s + e];
    return o;
  }
  // ds_read_b64_tr_b16 hands a lane 4 values that are consecutive along the rows
  template <int LD> static __device__ __forceinline__ col8 col(const E* tile, int k0, int n0, int lane) {
    const int r = lane & 15, gi = lane >> 4;
    const E* p = tile + (k0 + 4 * (gi >> 1) + (r >> 2)) * LD + n0 + 16 * (gi & 1) + 4 * (r & 3);
    union { struct { s16x4 a, b; } s; col8 v; } u;
    u.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
    u.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * LD));
    return u.v;
  }
};
template <> struct Mat<float> {
  typedef f32x4 vec;
  typedef f32x8 col8;
  static __device__ __forceinline__ f32x16 rows(vec a, vec b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ f32x16 cols(col8 a, col8 b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ col8 pack(const f32x16& x, int s) {
    col8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = x[8 * s + e];
    return o;
  }
  template <int LD> static __device__ __forceinline__ col8 col(const float* tile, int k0, int n0, int lane) {
    col8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = tile[(k0 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * LD + n0 + (lane & 31)];
    return o;
  }
};

// Rows of D columns in LDS.  The padding spreads rows over the banks: 16-bit rows of 304, 240 and 176 bytes start in different groups
// of 4 banks; fp32 rows are 8 (mod 16) floats apart, so that the two halves of a column read, 4 rows apart, take 32 banks each.
template <typename E, int D> struct Tile {
  static constexpr int VN = 16 / (int)sizeof(E), LD = D + (sizeof(E) == 2 ? 24 : 8), FRAGS = D / (2 * VN), BLOCKS = D / 32;
  typedef typename Mat<E>::vec vec;
  // columns 2 VN s + VN (lane/32) .. of row row0 + lane%32: an operand of the products over the columns
  static __device__ __forceinline__ vec frag(const E* tile, int row0, int s, int lane) {
    return *reinterpret_cast<const vec*>(tile + (row0 + (lane & 31)) * LD + 2 * VN * s + VN * (lane >> 5));
  }
  // The same of rows in memory; rows at or past `end` and columns past dd are zeros.
  static __device__ __forceinline__ void load_frags(vec (&f)[FRAGS], const E* __restrict__ head, int64_t ld, int row, int end, int lane, int dd) {
#pragma unroll
    for (int s = 0; s < FRAGS; ++s) {
      const int c = 2 * VN * s + VN * (lane >> 5);
      f[s] = vec{};
      if (row < end && c < dd) f[s] = *reinterpret_cast<const vec*>(head + row * ld + c);
    }
  }
  // A wave's accumulators, block by block of 32 columns, into the rows row0 + lane%32 below `end` by way of its own part of the LDS, so
  // that they leave as whole lines.
  static __device__ __forceinline__ void store(const f32x16 (&acc)[BLOCKS], float factor, E* lds, E* head, int64_t ld, int row0, int end, int lane, int dd,
                                               unsigned skip) {
    typedef E quad __attribute__((ext_vector_type(4)));
    wave_lds_order();
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        quad w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = from_f<E>(acc[b][4 * c + e] * factor);
        *reinterpret_cast<quad*>(lds + (lane & 31) * LD + 32 * b + 8 * c + 4 * (lane >> 5)) = w;
      }
    wave_lds_order();
    constexpr int P = D / VN;
#pragma unroll
    for (int i = 0; i < 32 * P / 64; ++i) {
      const int v = lane + 64 * i, r = v / P, c = v % P * VN;
      const vec w = *reinterpret_cast<const vec*>(lds + r * LD + c);
      if (row0 + r < end && c < dd && !(skip >> r & 1)) *reinterpret_cast<vec*>(head + (row0 + r) * ld + c) = w;
    }
  }
};

// ROWS rows on their way from memory to LDS through the registers of NT threads: fetch is issued before the products of the tile before, put
// comes after them.  Rows are read through a buffer descriptor of the tile's own, so that offsets inside it are 32 bits wide however far the
// rows lie apart; rows past the last one wanted and the columns past dd lie behind the descriptor's end and read as zeros.
template <typename E, int D, int ROWS, int NT> struct TileLoad {
  static constexpr int VN = Tile<E, D>::VN, P = D / VN, N = ROWS * P, NV = (N + NT - 1) / NT;
  u32x4 v[NV];
  __device__ __forceinline__ void fetch(const E* head, int64_t ld, int row0, int end, unsigned tid, int dd) {
    const int rows = min(end - row0, ROWS);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>(head + row0 * ld), 0,
                                                                        rows > 0 ? (int)(((rows - 1) * ld + dd) * sizeof(E)) : 0, 0x00020000);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int p = (int)tid + NT * i, r = p / P, c = p % P * VN;
      v[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, c < dd && (N % NT == 0 || p < N) ? (int)((r * (int)ld + c) * sizeof(E)) : (int)0x80000000, 0, 0);
    }
  }
  __device__ __forceinline__ void put(E* tile, unsigned tid) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int p = (int)tid + NT * i;
      if (N % NT == 0 || p < N) *reinterpret_cast<u32x4*>(tile + p / P * Tile<E, D>::LD + p % P * VN) = v[i];
    }
  }
};

// First and last of a wave's (or block's) tokens that have a range.  Ranges grow from token to token, so theirs are its union's ends (lo,
// hi) and what all of them share (all_lo, all_hi).
struct Span { int lo, hi, all_lo, all_hi; };
__device__ __forceinline__ Span span_of(int lo, int hi) {
  const unsigned long long live = __ballot(lo < hi);
  if (!live) return Span{0, 0, 0, 0};
  const int first = __ffsll(live) - 1, last = 63 - __clzll(live);
  return Span{__builtin_amdgcn_readlane(lo, first), __builtin_amdgcn_readlane(hi, last), __builtin_amdgcn_readlane(lo, last),
              __builtin_amdgcn_readlane(hi, first)};
}
__device__ __forceinline__ Span span_join(const Span& a, const Span& b) { return a.lo >= a.hi ? b : b.lo >= b.hi ? a : Span{a.lo, b.hi, b.all_lo, a.all_hi}; }
// Of `n` (at most 128) tokens from t0: the keys that they see, or the rows that see them.
template <bool ROWS> __device__ __forceinline__ Span block_span(const int32_t* ranges, int t0, int n, int T, int lane) {
  int lo[2], hi[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = lane + 64 * i;
    const int4 r = t < n && t0 + t < T ? doc_range((const int4*)ranges, t0 + t, T) : make_int4(0, 0, 0, 0);
    lo[i] = ROWS ? r.z : r.x;
    hi[i] = ROWS ? r.w : r.y;
  }
  return span_join(span_of(lo[0], hi[0]), span_of(lo[1], hi[1]));
}

// The scores of a block, in powers of two.  factor: what turns an entry of `s` into that: scale * log2 e where there is neither cap nor bias
// and s stays as the product left it, else 1.
//   capped: softcap tanh(u / softcap) = softcap - 2 softcap / (1 + exp(2 u / softcap)); 16-bit types take it so, with the hardware's
//   exp2 and reciprocal (absolute error softcap 2^-22, of weights that are then rounded to 2^-9 or 2^-12 of themselves); fp32 takes tanhf.
struct DocScale {
  float log2, cap, cap_log2, into_tanh, slope_log2;   // scale log2 e; softcap; softcap log2 e; 2 scale log2 e / softcap, or (fp32) scale / softcap; slope log2 e
  bool capped, biased;
  __device__ __forceinline__ float factor() const { return capped || biased ? 1.f : log2; }
};
template <typename E> __device__ __forceinline__ DocScale doc_scale(const DocAttn& a, int h) {
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  const bool capped = a.softcap > 0.f;
  return DocScale{a.scale * DOC_LOG2E, a.softcap, a.softcap * DOC_LOG2E, capped ? (sizeof(E) == 4 ? a.scale : 2.f * DOC_LOG2E * a.scale) / a.softcap : 0.f,
                  slope * DOC_LOG2E, capped, a.slopes != nullptr};
}
// tanh(u / softcap) of a product, as (1 - tanh) / 2 in 16-bit types
template <typename E> __device__ __forceinline__ float cap_part(const DocScale& c, float product) {
  if constexpr (sizeof(E) == 4) return tanhf(product * c.into_tanh);
  else return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(product * c.into_tanh));
}
template <typename E> __device__ __forceinline__ float cap_score(const DocScale& c, float part) {
  return sizeof(E) == 4 ? c.cap_log2 * part : fmaf(-2.f * c.cap_log2, part, c.cap_log2);
}
template <typename E> __device__ __forceinline__ float cap_slope(float part) {
  return sizeof(E) == 4 ? (1.f - part) * (1.f + part) : 4.f * part * (1.f - part);
}
// apart: of the lane's own token and the one that its register 0 stands for
__device__ __forceinline__ float bias_score(const DocScale& c, float apart, int r) { return -c.slope_log2 * fabsf(apart + (float)(8 * (r >> 2) + (r & 3))); }

template <typename E> __device__ __forceinline__ void doc_scores(f32x16& s, const DocScale& c, float apart) {
  if (c.capped) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = cap_score<E>(c, cap_part<E>(c, s[r]));
  } else if (c.biased) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] *= c.log2;
  }
  if (c.biased) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] += bias_score(c, apart, r);
  }
}
// Weights p = exp2(score - lse2[r]) into s, and p * (dp - delta[r]) * (the cap's slope) * factor into dp.  lse2 and delta: of the row that a register
// (dK/dV) or the lane (dQ) stands for.
template <typename E, typename F, typename G>
__device__ __forceinline__ void doc_weights(f32x16& s, f32x16& dp, const DocScale& c, float apart, float p_shift, float factor, F&& lse2, G&& delta) {
  if (!c.capped && !c.biased) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c.log2, p_shift - lse2(r)));
      dp[r] = s[r] * ((dp[r] - delta(r)) * factor);
    }
  } else if (!c.capped) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c.log2, p_shift - lse2(r)) + bias_score(c, apart, r));
      dp[r] = s[r] * ((dp[r] - delta(r)) * factor);
    }
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float part = cap_part<E>(c, s[r]);
      float x = cap_score<E>(c, part) + (p_shift - lse2(r));
      if (c.biased) x += bias_score(c, apart, r);
      s[r] = __builtin_amdgcn_exp2f(x);
      dp[r] = s[r] * ((dp[r] - delta(r)) * factor) * cap_slope<E>(part);
    }
  }
}

// Rows whose sums are not finite are computed again, one wave per row (attention_docs_rows.h).  In LDS, free by then: a row or two per wave, and
// the rows' bits per group of 32.
template <int NW> struct DocRedo { float rows[NW][256]; unsigned masks[NW]; };
template <int N> __device__ __forceinline__ float mark_of(const f32x16 (&x)[N]) {
  float mark[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) mark[r % 4] = mark_non_finite(mark[r % 4], x[i][r]);
  return (mark[0] + mark[1]) + (mark[2] + mark[3]);
}
// Publishes the rows of a group (writer: one wave per group); all waves of the workgroup call it.
template <int NW> __device__ __forceinline__ unsigned redo_rows(DocRedo<NW>& lds, int group, bool writer, bool bad) {
  const unsigned long long m = __ballot(bad);
  const unsigned rows = (unsigned)m | (unsigned)(m >> 32);
  if (writer) lds.masks[group] = rows;
  __syncthreads();
  return rows;
}
// The accumulators of `n` waves that share rows meet in the first one's, in the order of the waves.  red: (n - 1) * BLOCKS * 256 f32x4 ... of LDS
// that is free; the caller's barrier frees it again.
template <int BLOCKS> __device__ __forceinline__ void merge_waves(f32x16 (&acc)[BLOCKS], f32x4* red, int which, int n, int lane) {
  if (which > 0) {
    f32x4* to = red + (which - 1) * BLOCKS * 4 * 64;
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) to[(i * 4 + c) * 64 + lane] = f32x4{acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]};
  }
  __syncthreads();
  if (which == 0) {
    for (int w = 1; w < n; ++w)
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const f32x4 o = red[((w - 1) * BLOCKS * 4 + i * 4 + c) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][4 * c + e] += o[e];
        }
  }
  __syncthreads();
}

}  // namespace
}  // namespace zs
