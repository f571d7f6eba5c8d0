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

// What a lane reads 16 bytes at a time (vec), and 8 rows of a column (col8): of the rows 16 s + 4 (lane/32) + {0 .. 3, 8 .. 11}, in the order
// of the accumulators 8 s .. 8 s + 7.
template <typename E> struct Mat {
  typedef typename Vec<E>::type vec;
  typedef vec col8;
  static __device__ __forceinline__ f32x16 mma(vec a, vec b, f32x16 c) {
    if constexpr (__is_same(E, bf16)) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 rows(vec a, vec b, f32x16 c) { return mma(a, b, c); }
  static __device__ __forceinline__ f32x16 cols(col8 a, col8 b, f32x16 c) { return mma(a, b, c); }
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
};
template <typename E> __device__ __forceinline__ typename Mat<E>::col8 pack(const f32x16& x, int s) {
  typename Mat<E>::col8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = from_f<E>(x[8 * s + e]);
  return o;
}

typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ unsigned lds_address(const void* p) { return (unsigned)(uintptr_t)(const lds_char*)p; }
template <typename T> __device__ __forceinline__ T lds_read(unsigned at) { return *(const __attribute__((address_space(3))) T*)(uintptr_t)at; }

// Tiles of rows in LDS, D columns wide.  They come straight from memory (buffer loads into LDS), a wave's load bringing 1 KB: 8 rows by 128
// bytes, lane l the piece of 16 bytes that belongs at 16 l.  Piece p of row r of such a square sits at position p ^ turn(r) of the row, which
// the lanes arrange by what they load; squares of 8 rows are followed by a gap of 128 bytes.  Then the 16 rows that one cycle of a fragment
// read touches lie in 16 different groups of 4 banks, and so do the 4 rows x 64 bytes of half a transposing read.  Of a fragment's
// address only the place inside a square depends on the lane: four values for row fragments and two (fp32: four) for columns.  Measured on the forward
// of 8192 tokens: 0.8 M of 70.6 M LDS cycles are conflicts; tiles that came through registers (two dozen of them) into padded rows 619 us, these 555.
template <typename E, int D> struct Tile {
  static constexpr int SZ = (int)sizeof(E), VN = 16 / SZ, FRAGS = D / (2 * VN), BLOCKS = D / 32, SQUARES = (D * SZ + 127) / 128;
  static constexpr int OCTET = SQUARES * 1024 + 128;   // bytes of 8 rows
  static constexpr int bytes(int rows) { return rows / 8 * OCTET; }
  static constexpr int COLS = SZ == 4 ? 4 : 2;
  typedef typename Mat<E>::vec vec;
  typedef typename Mat<E>::col8 col8;

  static __device__ __forceinline__ unsigned turn(unsigned r) { return (r & 1) | (r & 2) << 1 | (r & 4) >> 1; }
  static __device__ __forceinline__ unsigned place(unsigned row, unsigned piece) { return row * 128 + ((piece ^ turn(row)) << 4); }

  // A lane's places, on top of an address in LDS.
  struct Lane {
    unsigned row[4], col[COLS];
    __device__ __forceinline__ Lane(unsigned base, int lane) {
#pragma unroll
      for (int s = 0; s < 4; ++s) row[s] = base + (lane & 31) / 8 * OCTET + place(lane & 7, 2 * s + (lane >> 5));
#pragma unroll
      for (int i = 0; i < COLS; ++i)
        col[i] = base + (SZ == 4 ? place(4 * (lane >> 5) + i, (lane & 31) >> 2) + 4 * (lane & 3)
                                 : place(4 * (lane >> 5) + (lane & 15) / 4, 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1));
    }
    __device__ __forceinline__ void move(int by) {
#pragma unroll
      for (int s = 0; s < 4; ++s) row[s] += by;
#pragma unroll
      for (int i = 0; i < COLS; ++i) col[i] += by;
    }
    // columns 2 VN s + VN (lane/32) .. of row row0 + lane%32: an operand of the products over the columns
    __device__ __forceinline__ vec frag(int tile, int row0, int s) const { return lds_read<vec>(row[s & 3] + (tile + row0 / 8 * OCTET + (s >> 2) * 1024)); }
    // column 32 b + lane%32 of 16 rows from row0 on: an operand of the products over the rows
    __device__ __forceinline__ col8 column(int tile, int row0, int b) const {
      if constexpr (SZ == 4) {
        col8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = lds_read<float>(col[e & 3] + (tile + (row0 / 8 + (e >> 2)) * OCTET + b * 1024));
        return o;
      } else {   // ds_read_b64_tr_b16 hands a lane 4 values that are consecutive along the rows
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const unsigned at = col[b & 1] + (tile + row0 / 8 * OCTET + (b >> 1) * 1024);
        union { struct { s16x4 a, b; } s; col8 v; } u;
        u.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)at);
        u.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(at + OCTET));
        return u.v;
      }
    }
  };

  // Row fragments from memory; rows at or past `end` and columns past dd are zeros.
  static __device__ __forceinline__ void load_frags(vec (&f)[FRAGS], const E* __restrict__ head, int64_t ld, int row, int end, int lane, int dd) {
#pragma unroll
    for (int s = 0; s < FRAGS; ++s) {
      const int c = 2 * VN * s + VN * (lane >> 5);
      f[s] = vec{};
      if (row < end && c < dd) f[s] = *reinterpret_cast<const vec*>(head + row * ld + c);
    }
  }
  // A wave's accumulators, block by block of 32 columns, into the rows row0 + lane%32 below `end` by way of its own part of the LDS (STORE
  // bytes), so that they leave as whole lines.  skip: rows that stay as they are.
  static constexpr int LD = D + (SZ == 2 ? 24 : 8), STORE = 32 * LD * SZ;
  static __device__ __forceinline__ void store(const f32x16 (&acc)[BLOCKS], float factor, char* lds, E* head, int64_t ld, int row0, int end, int lane,
                                               int dd, unsigned skip) {
    typedef E quad __attribute__((ext_vector_type(4)));
    E* rows = reinterpret_cast<E*>(lds);
    wave_lds_order();
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        quad w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = from_f<E>(acc[b][4 * c + e] * factor);
        *reinterpret_cast<quad*>(rows + (lane & 31) * LD + 32 * b + 8 * c + 4 * (lane >> 5)) = w;
      }
    wave_lds_order();
    constexpr int P = D / VN;
#pragma unroll
    for (int i = 0; i < 32 * P / 64; ++i) {
      const int v = lane + 64 * i, r = v / P, c = v % P * VN;
      const vec w = *reinterpret_cast<const vec*>(rows + r * LD + c);
      if (row0 + r < end && c < dd && !(skip >> r & 1)) *reinterpret_cast<vec*>(head + (row0 + r) * ld + c) = w;
    }
  }
};

// Brings ROWS rows into LDS by NW waves.  The rows are read through a buffer descriptor of the tile's own, so that offsets inside it are 32 bits wide however
// far the rows lie apart; rows at or past `end` and the columns past dd lie behind the descriptor's end and arrive as zeros.  tile_wait, before the
// barrier that publishes a tile, waits for what a wave has under way.
template <typename E, int D, int ROWS, int NW> struct TileLoad {
  typedef Tile<E, D> TL;
  static constexpr int N = ROWS / 8 * TL::SQUARES / NW;
  static_assert(N * NW * 8 == ROWS * TL::SQUARES, "");
  unsigned at[TL::SQUARES];   // of a lane's piece in the first 8 rows
  int ld, width;              // elements of a row, bytes of a head's part of it
  __device__ __forceinline__ TileLoad(int64_t stride, int lane, int dd) : ld((int)stride), width(dd * TL::SZ) {
#pragma unroll
    for (int q = 0; q < TL::SQUARES; ++q) {
      const int c = (8 * q + (int)((lane & 7) ^ TL::turn(lane >> 3))) * TL::VN;
      at[q] = c < dd ? (unsigned)((lane >> 3) * ld + c) * TL::SZ : 0x80000000u;
    }
  }
  __device__ __forceinline__ void fetch(unsigned lds, const E* head, int row0, int end, int wave) const {
    const int rows = min(end - row0, ROWS);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>(head + (int64_t)row0 * ld), 0,
                                                                        rows > 0 ? (rows - 1) * ld * TL::SZ + width : 0, 0x00020000);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      // a wave's loads lie in one column of squares where the waves are as many as these columns, or a multiple
      const int sq = wave + NW * i, oct = sq / TL::SQUARES, q = sq % TL::SQUARES;
      unsigned from = at[0];
#pragma unroll
      for (int k = 1; k < TL::SQUARES; ++k) from = q == k ? at[k] : from;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(uintptr_t)(lds + oct * TL::OCTET + q * 1024), 16,
                                               from + (unsigned)(8 * oct * ld * TL::SZ), 0, 0, 0);
    }
  }
};
__device__ __forceinline__ void tile_wait() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
  __builtin_amdgcn_sched_barrier(0);
}

// Row fragments of 32 rows by way of LDS of the wave's own (Tile::bytes(32)), so that they come as whole lines: the lanes of a fragment load lie in 32
// rows, and the address unit takes four times as long for their pieces.  us, bf16, heads of 128, by fragments : by lines in all kernels: 1024 packed tokens,
// 16 heads, forward 18.7 : 17.8, backward 46.3 : 41.7; one document of 2048 tokens, 8 heads 28.0 : 27.5 and 70.0 : 65.1.
template <typename E, int D, typename V, int N>
__device__ __forceinline__ void load_frags_by_lines(V (&f)[N], unsigned lds, const E* head, int64_t ld, int row0, int end, int lane, int dd) {
  const TileLoad<E, D, 32, 1> load(ld, lane, dd);
  const typename Tile<E, D>::Lane at(lds, lane);
  wave_lds_order();   // the rows before have been read
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): they have arrived before others take their place
  __builtin_amdgcn_sched_barrier(0);
  load.fetch(lds, head, row0, end, 0);
  tile_wait();
  wave_lds_order();
#pragma unroll
  for (int s = 0; s < N; ++s) f[s] = at.frag(0, 0, s);
}

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
// Of `n` (at most 64 N) tokens from t0: the keys that they see, or the rows that see them.
template <bool ROWS, int N> __device__ __forceinline__ Span block_span(const int32_t* ranges, int t0, int n, int T, int lane) {
  int lo[N], hi[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int t = lane + 64 * i;
    const int4 r = t < n && t0 + t < T ? doc_range((const int4*)ranges, t0 + t, T) : make_int4(0, 0, 0, 0);
    lo[i] = ROWS ? r.z : r.x;
    hi[i] = ROWS ? r.w : r.y;
  }
  Span all = span_of(lo[0], hi[0]);
#pragma unroll
  for (int i = 1; i < N; ++i) all = span_join(all, span_of(lo[i], hi[i]));
  return all;
}
// The rank-th longest of `blocks` (at most 256) blocks of `rows` (at most 128) tokens, by the keys that they see or the rows that see them, in 128
// steps of 128 (above 127 * 128 tokens 256) and, where equal, the earlier one first. Which tokens begin a document is known on the device only, so
// each workgroup finds its block by itself: the blocks' numbers (length, then place) lie four to a lane, and the one with `rank` larger ones is found
// bit by bit, by counting.
template <bool ROWS> __device__ __forceinline__ int heavy_block(const int32_t* ranges, int T, int rows, int blocks, int rank, int lane) {
  int number[4];
  const int step = T <= 127 * 128 ? 7 : 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = lane + 64 * i;
    number[i] = -1;
    if (b < blocks) {
      const int4 first = doc_range((const int4*)ranges, b * rows, T), last = doc_range((const int4*)ranges, min(b * rows + rows, T) - 1, T);
      const int4 &a = first.x < first.y ? first : last, &z = last.x < last.y ? last : first;   // of a document, where the block has padding before or behind it
      const int span = ROWS ? z.w - a.z : z.y - a.x;
      number[i] = min(max((span + (1 << step) - 1) >> step, 0), 127) << 8 | (255 - b);
    }
  }
  int found = 0;
  for (int bit = 1 << 14; bit; bit >>= 1) {
    const int above = found | bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += __popcll(__ballot(number[i] >= above));
    if (n > rank) found = above;
  }
  return 255 - (found & 255);
}

// The scores of a block, in powers of two: what a register holds after doc_scores, times f, plus g.  MODE says which of cap and bias a call has.
//   plain: the product as it is, f = scale log2 e.
//   capped: softcap tanh(u / softcap) = softcap - 2 softcap r, r = 1 / (1 + exp(2 u / softcap)).  16-bit types keep r (so the largest score is the
//   smallest register), from the hardware's exp2 and reciprocal: an absolute error of softcap 2^-22, of weights that are then rounded to 2^-9 or 2^-12
//   of themselves.  fp32 keeps tanh_f.
//   biased: with the bias in.
// The vector units bound a capped kernel, so its additions are folded: g goes with the reference or the log-sum-exp that is subtracted anyway, and the
// cap's slope 1 - tanh^2 = 4 (r - r^2) leaves its 4 (DOC_UNIT) to a factor that is there anyway: the gradients' last one (DOC_SLOPE), or in half, where a
// quarter of a score gradient may lie below the normal numbers, the one that it is multiplied by before its rounding.
enum DocMode { DOC_PLAIN = 0, DOC_CAP = 1, DOC_BIAS = 2 };   // or-ed
template <typename E, int MODE> constexpr bool DOC_FALLS = MODE == DOC_CAP && sizeof(E) == 2;   // f < 0
template <typename E, int MODE> constexpr float DOC_UNIT = (MODE & DOC_CAP) && sizeof(E) == 2 ? 4.f : 1.f;
template <typename E, int MODE> constexpr float DOC_SLOPE = __is_same(E, f16) ? 1.f : DOC_UNIT<E, MODE>;
struct DocScale {
  float log2, cap, into_tanh, slope, g;   // scale log2 e; of tanh or r; 2 scale log2 e / softcap, or (fp32) scale / softcap; slope log2 e; see above
  template <int MODE> __device__ __forceinline__ float f() const { return MODE == DOC_PLAIN ? log2 : MODE == DOC_CAP ? cap : 1.f; }
};
template <typename E, int MODE> __device__ __forceinline__ DocScale doc_scale(const DocAttn& a, int h) {
  constexpr bool CAP = MODE & DOC_CAP, HALF_SIZE = sizeof(E) == 2;
  const float cap = a.softcap * DOC_LOG2E;
  return DocScale{a.scale * DOC_LOG2E, HALF_SIZE ? -2.f * cap : cap, CAP ? (HALF_SIZE ? 2.f * DOC_LOG2E * a.scale : a.scale) / a.softcap : 0.f,
                  MODE & DOC_BIAS ? a.slopes[h] * DOC_LOG2E : 0.f, CAP && HALF_SIZE ? cap : 0.f};
}
// tanh within 1.9e-7 of itself (the largest of all floats from 2^-20 on, in 0.6 .. 1; below 0.5 6.3e-8), without branches: below 0.6 an odd
// polynomial (fitted by least squares in the relative error, which is 4e-9 with these coefficients), above from the exponential, whose cancellation
// is harmless there. 12 vector and 2 transcendental instructions.
__device__ __forceinline__ float tanh_f(float u) {
  const float z = u * u;
  float p = 0.0022269718f;
  p = fmaf(p, z, -0.0082627423f);
  p = fmaf(p, z, 0.021732720f);
  p = fmaf(p, z, -0.053952165f);
  p = fmaf(p, z, 0.13333246f);
  p = fmaf(p, z, -0.33333331f);
  const float t = fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.f * DOC_LOG2E * fabsf(u))), 1.f);
  return fabsf(u) < 0.6f ? fmaf(u * z, p, u) : copysignf(t, u);
}
// tanh(u / softcap) of a product, or r.
template <typename E> __device__ __forceinline__ float cap_part(const DocScale& c, float product) {
  if constexpr (sizeof(E) == 4) return tanh_f(product * c.into_tanh);
  else return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(product * c.into_tanh));
}
// The bias.  apart: of the lane's own token and the one that its register 0 stands for
__device__ __forceinline__ float bias_score(const DocScale& c, float apart, int r) { return -c.slope * fabsf(apart + (float)(8 * (r >> 2) + (r & 3))); }
template <typename E, int MODE> __device__ __forceinline__ void doc_scores(f32x16& s, const DocScale& c, float apart) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if constexpr (MODE & DOC_CAP) s[r] = cap_part<E>(c, s[r]);
    if constexpr (MODE & DOC_BIAS) s[r] = fmaf(s[r], MODE & DOC_CAP ? c.cap : c.log2, bias_score(c, apart, r));
  }
}
// Weights p = exp2(score - lse2) into s, and p * (dp - delta) * (the cap's slope / DOC_UNIT) * (half: factor) into dp.  lse2(c), less g, and delta(c): of the rows
// (dK/dV) that the registers 4 c .. 4 c + 3 stand for, or of the lane's own (dQ).
template <typename E, int MODE, typename F, typename G>
__device__ __forceinline__ void doc_weights(f32x16& s, f32x16& dp, const DocScale& c, float apart, float factor, F&& lse2, G&& delta) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f32x4 l = lse2(g), d = delta(g);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * g + e;
      const float part = MODE & DOC_CAP ? cap_part<E>(c, s[r]) : s[r];
      float x = fmaf(part, MODE & DOC_CAP ? c.cap : c.log2, -l[e]);
      if constexpr (MODE & DOC_BIAS) x += bias_score(c, apart, r);
      s[r] = __builtin_amdgcn_exp2f(x);
      float ds = s[r] * (dp[r] - d[e]);
      if constexpr (MODE & DOC_CAP) ds *= fmaf(-part, part, sizeof(E) == 4 ? 1.f : part);
      dp[r] = __is_same(E, f16) ? ds * factor : ds;
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
// The accumulators of `n` waves that share rows meet in the first one's, in the order of the waves.  red: (n - 1) * BLOCKS * 256 f32x4 of LDS
// that is free, and free again when the call returns.
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
