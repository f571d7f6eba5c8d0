// Attention inside packed documents on the matrix cores, in one pass over the keys, forward and backward, of one element type (bf16, half and float each
// build it: attention_docs_*.hip).
//
// The T x T scores are never stored.  A block of rows reads only the keys that its documents' ranges span, from the first of them on:
// tiles begin at that key, whatever its number, and rows past the span's end read as zeros.  A wave skips tiles that none of its rows
// sees, and compares row by row only where not all of its rows see the whole tile.  Query heads that share a key head share a workgroup,
// which then holds 32 rows of four heads instead of 128 rows of one and walks fewer keys that some of its rows do not see.
//
// The backward is two kernels without atomics: dQ by blocks of rows, dK and dV by blocks of keys over all the query heads of a key head;
// both form the weights again from the saved log-sum-exp.
//
// 16-bit types round the weights P and the score gradients dS to their type for the second product: half a step of each term, about what the
// result's own rounding costs.  Half's range is helped by powers of two, taken out at the end: P goes in times 2^7 or 2^14, dS relative to the
// largest dO of its row (dQ), or of the rows so far that see its key (dK): a key's own, or another document's dO would coarsen it.
#pragma once
#include "attention_docs_tiles.h"

namespace zs {
namespace {

template <typename E> constexpr bool HALF = __is_same(E, f16);
template <typename E> constexpr float P_LAG = HALF<E> ? 7.f : 0.f;     // forward: weights are at most 2^(8 + lag)
template <typename E> constexpr float P_SHIFT = HALF<E> ? 14.f : 0.f;  // backward: weights times 2^shift
// 2^-e for the exponent e of x > 0, within what halves times it can use; 1 for 0, inf and NaN
__device__ __forceinline__ float unit_of(float x) {
  const int e = (int)((__float_as_uint(x) >> 23) & 255) - 127;
  return e > 60 || e < -60 ? 1.f : __uint_as_float((unsigned)(127 - e) << 23);
}

// Blocks of rows, all heads of a block before the next one; key heads in the fastest place, so that the blocks of a key head stay on an XCD where
// there are 8 of them and find its keys in its L2.  The longest blocks come first: by their ranges (a.sorted), or, where they are too many to be ordered
// (over 256) or all begin at once, the last ones, which are the longest of one causal document; of several they are in no order.
struct DocBlock { int block, kv, h; };
__device__ __forceinline__ DocBlock row_block(const DocAttn& a, int workgroup, int heads, int rows, int lane) {   // heads of a key head in a workgroup, rows of a block
  const int group = a.nh / a.nkv, sets = a.nkv * (group / heads), blocks = (a.T + rows - 1) / rows;
  const int set = workgroup % sets, kv = set % a.nkv, rank = workgroup / sets;
  return DocBlock{a.sorted ? heavy_block<false>(a.ranges, a.T, rows, blocks, rank, lane) : blocks - 1 - rank, kv, kv * group + set / a.nkv * heads};
}

// Calls of their own, not inlined, so that the registers of the kernels' loops are not planned around them. A kernel is given as many as the calls
// need all the same: heads of 64 forward 150 (without the call 102 to 126, four waves per SIMD instead of three), dQ 179 and 168 (bf16, half; 122 to
// 145), dK/dV 209 and 198 (160 to 179, 182 to 189); heads of 96 and 128 need more themselves.
template <typename E, int NW>
__device__ __attribute__((noinline)) void redo_fwd(DocRedo<NW>* redo, int groups, int row_groups, int t0, const int32_t* ranges, int T, int d, const E* q,
                                                   int64_t ldq, const E* k, const E* v, int64_t ldkv, float scale, float softcap, const float* slopes,
                                                   E* o, int64_t ldo) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for_dealt_rows(redo->masks, groups, NW, wave, [&](int g, int r) {
    const int h = g / row_groups, i = t0 + 32 * (g % row_groups) + r;
    const int4 range = doc_range((const int4*)ranges, i, T);
    doc_fwd_row<E>(redo->rows[wave], i, range.x, range.y, d, DocRows<E>{q + h * d, ldq}, DocRows<E>{k, ldkv}, DocRows<E>{v, ldkv}, scale,
                   DocScore{softcap, slopes ? slopes[h] : 0.f}, lane, [&](int c, float x) { o[i * ldo + h * d + c] = from_f<E>(x); });
  });
}

// ------------------------------------------------------------------------------------------ forward
// NW waves in groups that have 32 rows of their own.  KS = 1: a wave to a group, which walks all keys of a tile; two workgroups of four waves to a CU.
// KS = 2, 4: that many waves share a group's rows, each takes its part of a tile's keys, and their sums meet at the end: for few rows.
// What bounds it: a long document's 32 x 32 blocks cost 16 matrix instructions of 32 cycles (heads of 128) and about as many vector cycles (exponentials,
// maximum, sums, conversion; with a cap twice that), which two waves per SIMD overlap little: of 8192 tokens after a prefix, 32 heads, 52 % of the
// SIMDs' cycles are matrix and 45 % vector instructions at 1.05 PFLOP/s (a library product of 8192^3: 1.11).  Two waves held half a step apart by
// barriers, one at its products while the other forms weights, were slower (529 -> 639 us), and so were the next tile's scores issued between this one's
// exponentials (531 -> 564), and tiles without the maximum, which is formed again only where the sums show that it has moved (574 -> 595: the sums' test
// keeps the exponentials apart from the products behind it).  Raised wave priority around the products: no difference.
template <typename E, int D, int MODE, int NW, int KS, int ROWS>
__global__ __launch_bounds__(64 * NW, NW == 8 || KS == 1 ? 2 : 1) void doc_fwd_kernel(DocAttn a, int heads) {
  typedef Tile<E, D> TL;
  typedef Mat<E> M;
  constexpr int GROUPS = NW / KS, SUB = ROWS / 32 / KS, TILE = TL::bytes(ROWS);
  constexpr bool LINES = 2 * ROWS >= 32 * NW;   // q comes by whole lines through the second buffer, where that holds the waves' rows
  constexpr float LAG = P_LAG<E>;
  constexpr size_t LOOP = 4 * TILE, END = sizeof(DocRedo<NW>) + 16 + GROUPS * TL::STORE;   // two buffers of keys and values
  __shared__ __align__(16) char smem_raw[LOOP > END ? LOOP : END];
  static_assert((LOOP > END ? LOOP : END) >= (size_t)(KS - 1) * GROUPS * TL::BLOCKS * 4 * 64 * 16, "");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ks = wave / GROUPS, grp = wave % GROUPS, row_groups = GROUPS / heads, h_in = grp / row_groups, dd = a.d;
  const DocBlock blk = row_block(a, blockIdx.x, heads, 32 * row_groups, lane);
  const int t0 = blk.block * 32 * row_groups, w0 = t0 + 32 * (grp % row_groups), my_q = w0 + (lane & 31), h = blk.h + h_in;
  const E* qh = (const E*)a.q + h * dd;
  const E *kh = (const E*)a.k + blk.kv * dd, *vh = (const E*)a.v + blk.kv * dd;
  const Span all = block_span<false, (32 * GROUPS + 63) / 64>(a.ranges, t0, 32 * row_groups, a.T, lane);
  const int4 range = my_q < a.T ? doc_range((const int4*)a.ranges, my_q, a.T) : make_int4(0, 0, 0, 0);
  typename M::vec qf[TL::FRAGS];
  if constexpr (!LINES) TL::load_frags(qf, qh, a.ldq, my_q, a.T, lane, dd);
  const DocScale sc = doc_scale<E, MODE>(a, h);
  const int lo = range.x, seen = max(range.y - range.x, 0);   // keys
  const Span mine = span_of(range.x, range.y);
  const int tiles = (all.hi - all.lo + ROWS - 1) / ROWS;

  const unsigned smem = lds_address(smem_raw);
  const TileLoad<E, D, ROWS, NW> load(a.ldkv, lane, dd);
  auto fetch = [&](unsigned to, int row0) {
    load.fetch(to, kh, row0, all.hi, wave);
    load.fetch(to + TILE, vh, row0, all.hi, wave);
  };
  typename TL::Lane at(smem + TL::bytes(ks * 32 * SUB), lane);
  f32x16 oacc[TL::BLOCKS];
#pragma unroll
  for (int i = 0; i < TL::BLOCKS; ++i) oacc[i] = f32x16{};
  float m = -INFINITY, l = 0.f;   // the reference of the weights, less g, and the sum of the lane's own
  if (tiles > 0) {
    fetch(smem, all.lo);
    if constexpr (LINES) load_frags_by_lines<E, D>(qf, smem + 2 * TILE + wave * TL::bytes(32), qh, a.ldq, w0, a.T, lane, dd);
    tile_wait();
    __syncthreads();
  }
  const float f = sc.f<MODE>(), MASKED = DOC_FALLS<E, MODE> ? INFINITY : -INFINITY;
  for (int t = 0; t < tiles; ++t) {
    const int key0 = all.lo + t * ROWS;
    if (t + 1 < tiles) fetch(smem + ((t + 1) & 1) * 2 * TILE, key0 + ROWS);   // that buffer was last read before the barrier that ended the iteration before
    const int kb = key0 + ks * 32 * SUB;
    if (kb < mine.hi && kb + 32 * SUB > mine.lo) {
      f32x16 s[SUB];
#pragma unroll
      for (int j = 0; j < SUB; ++j) {
        s[j] = f32x16{};
#pragma unroll
        for (int c = 0; c < TL::FRAGS; ++c) s[j] = M::rows(at.frag(0, 32 * j, c), qf[c], s[j]);
      }
#pragma unroll
      for (int j = 0; j < SUB; ++j) doc_scores<E, MODE>(s[j], sc, (float)(kb + 32 * j + 4 * (lane >> 5) - my_q));
      if (kb < mine.all_lo || kb + 32 * SUB > mine.all_hi) {   // not every row sees every key
#pragma unroll
        for (int j = 0; j < SUB; ++j) {
          const int from = kb + 32 * j + 4 * (lane >> 5) - lo;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((unsigned)(from + 8 * (r >> 2) + (r & 3)) >= (unsigned)seen) s[j][r] = MASKED;
        }
      }
      float mx = MASKED;   // of the registers; then the largest score, less g
#pragma unroll
      for (int j = 0; j < SUB; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = DOC_FALLS<E, MODE> ? fminf(mx, s[j][r]) : fmaxf(mx, s[j][r]);
      mx *= f;
      // The reference moves only when some row's maximum has outgrown it by 2^8: weights are at most 2^(8 + LAG), the sums and the result refer to the
      // same reference whenever it moves.  The two lanes of a row share the reference, but meet only here, and their sums at the end.
      if (__any(seen > 0 && mx > m + (8.f + LAG))) {
        const float mn = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32, 64)) - LAG), alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
        l *= alpha;
        m = mn;
#pragma unroll
        for (int i = 0; i < TL::BLOCKS; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[i][r] *= alpha;
      }
      const float ref = m == -INFINITY ? 0.f : m;   // no key seen so far: every weight is exp2(-inf)
      float part[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < SUB; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[j][r], f, -ref));
          s[j][r] = p;
          part[r & 1] += p;
        }
      l += part[0] + part[1];
#pragma unroll
      for (int j = 0; j < SUB; ++j)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const typename M::col8 pf = pack<E>(s[j], u);
#pragma unroll
          for (int b = 0; b < TL::BLOCKS; ++b) oacc[b] = M::cols(at.column(TILE, 32 * j + 16 * u, b), pf, oacc[b]);
        }
    }
    tile_wait();
    at.move(t & 1 ? -2 * TILE : 2 * TILE);
    __syncthreads();
  }
  l += __shfl_xor(l, 32, 64);
  if constexpr (KS > 1) {
    float* stat = reinterpret_cast<float*>(smem_raw) + grp * KS * 64;   // [GROUPS][KS][m | l][32]
    if (lane < 32) {
      stat[ks * 64 + lane] = m;
      stat[ks * 64 + 32 + lane] = l;
    }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < KS; ++w) top = fmaxf(top, stat[w * 64 + (lane & 31)]);
    const float ref = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f(m - ref);
    l = 0.f;
#pragma unroll
    for (int w = 0; w < KS; ++w) l += stat[w * 64 + 32 + (lane & 31)] * __builtin_amdgcn_exp2f(stat[w * 64 + (lane & 31)] - ref);
    m = top;
#pragma unroll
    for (int i = 0; i < TL::BLOCKS; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[i][r] *= alpha;
    __syncthreads();
    merge_waves<TL::BLOCKS>(oacc, reinterpret_cast<f32x4*>(smem_raw) + grp * (KS - 1) * TL::BLOCKS * 4 * 64, ks, KS, lane);
  }
  const bool live = seen > 0 && my_q < a.T;
  DocRedo<NW>& redo = *reinterpret_cast<DocRedo<NW>*>(smem_raw);
  const unsigned again = redo_rows<NW>(redo, grp, ks == 0, ks == 0 && live && !(mark_of(oacc) + l * 0.f == 0.f));
  if (ks == 0) {
    if (!live) {
#pragma unroll
      for (int i = 0; i < TL::BLOCKS; ++i) oacc[i] = f32x16{};
    }
    TL::store(oacc, live ? 1.f / l : 0.f, smem_raw + (sizeof(redo) + 15) / 16 * 16 + grp * TL::STORE, (E*)a.o + h * dd, a.ldo, w0, a.T,
              lane, dd, again);
    if (lane < 32 && my_q < a.T)
      a.lse[(int64_t)h * a.T + my_q] = live ? (float)(((double)m + (double)sc.g) * 0.6931471805599453 + (double)logf(l)) : -INFINITY;
  }
  if (__builtin_expect(any_row(redo.masks, GROUPS, lane), 0))
    redo_fwd<E, NW>(&redo, GROUPS, row_groups, t0, a.ranges, a.T, dd, (const E*)a.q + blk.h * dd, a.ldq, kh, vh, a.ldkv, a.scale, a.softcap,
                    a.slopes ? a.slopes + blk.h : nullptr, (E*)a.o + blk.h * dd, a.ldo);
}

// ------------------------------------------------------------------------------------------ dQ
// dQ^T += K^T dS^T, dS^T = P^T (dP^T - delta), dP^T = V dO^T.  Waves as in the forward; the one that has a row's dO forms its delta = dO.o and leaves
// it, and in half the row's largest |dO|, for the other kernel.
template <typename E, int NW>
__device__ __attribute__((noinline)) void redo_dq(DocRedo<NW>* redo, int groups, int row_groups, int t0, const int32_t* ranges, int T, int d, const E* q,
                                                  int64_t ldq, const E* k, const E* v, int64_t ldkv, const E* dout, int64_t ldo, const float* lse,
                                                  const float* delta, float scale, float softcap, const float* slopes, E* dq, int64_t lddq) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for_dealt_rows(redo->masks, groups, NW, wave, [&](int g, int r) {
    const int h = g / row_groups, i = t0 + 32 * (g % row_groups) + r;
    const int4 range = doc_range((const int4*)ranges, i, T);
    doc_dq_row<E>(redo->rows[wave], i, range.x, range.y, d, DocRows<E>{q + h * d, ldq}, DocRows<E>{k, ldkv}, DocRows<E>{v, ldkv},
                  DocRows<E>{dout + h * d, ldo}, lse[(int64_t)h * T + i], delta[(int64_t)h * T + i], scale, DocScore{softcap, slopes ? slopes[h] : 0.f}, lane,
                  [&](int c, float x) { dq[i * lddq + h * d + c] = from_f<E>(x); });
  });
}

template <typename E, int D, int NW, int KS, int ROWS, int NBUF> constexpr size_t dq_lds() {
  typedef Tile<E, D> TL;
  constexpr size_t LOOP = 2 * NBUF * TL::bytes(ROWS), END = sizeof(DocRedo<NW>) + 16 + NW / KS * TL::STORE,   // [NBUF][keys | values]
                   MERGE = (size_t)(KS - 1) * (NW / KS) * TL::BLOCKS * 4 * 64 * 16;
  return LOOP > END ? (LOOP > MERGE ? LOOP : MERGE) : END > MERGE ? END : MERGE;
}
template <typename E, int D, int MODE, int NW, int KS, int ROWS, int NBUF>
__device__ __forceinline__ void dq_block(char* smem_raw, const DocAttn& a, int workgroup, int heads) {
  typedef Tile<E, D> TL;
  typedef Mat<E> M;
  constexpr int GROUPS = NW / KS, SUB = ROWS / 32 / KS, TILE = TL::bytes(ROWS);
  // q, dout and o come by whole lines through the second buffer, where there is one and it holds the waves' rows.
  constexpr bool LINES = NBUF == 2 && 2 * ROWS >= 32 * NW;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ks = wave / GROUPS, grp = wave % GROUPS, row_groups = GROUPS / heads, h_in = grp / row_groups, dd = a.d;
  const DocBlock blk = row_block(a, workgroup, heads, 32 * row_groups, lane);
  const int t0 = blk.block * 32 * row_groups, w0 = t0 + 32 * (grp % row_groups), my_q = w0 + (lane & 31), h = blk.h + h_in;
  const E *kh = (const E*)a.k + blk.kv * dd, *vh = (const E*)a.v + blk.kv * dd;
  const Span all = block_span<false, (32 * GROUPS + 63) / 64>(a.ranges, t0, 32 * row_groups, a.T, lane);
  const int4 range = my_q < a.T ? doc_range((const int4*)a.ranges, my_q, a.T) : make_int4(0, 0, 0, 0);
  const int lo = range.x, seen = max(range.y - range.x, 0);
  const bool live = seen > 0 && my_q < a.T;
  typename M::vec qf[TL::FRAGS], dof[TL::FRAGS];
  if constexpr (!LINES) {
    TL::load_frags(qf, (const E*)a.q + h * dd, a.ldq, my_q, a.T, lane, dd);
    TL::load_frags(dof, (const E*)a.dout + h * dd, a.ldo, my_q, a.T, lane, dd);
  }
  const int64_t stat = (int64_t)h * a.T + min(my_q, a.T - 1);
  const DocScale sc = doc_scale<E, MODE>(a, h);
  const float lse2 = live ? fmaf(a.lse[stat], DOC_LOG2E, -sc.g) : 0.f;
  const Span mine = span_of(range.x, range.y);
  const int tiles = (all.hi - all.lo + ROWS - 1) / ROWS;
  const unsigned smem = lds_address(smem_raw);
  const TileLoad<E, D, ROWS, NW> load(a.ldkv, lane, dd);
  auto fetch = [&](unsigned to, int row0) {
    load.fetch(to, kh, row0, all.hi, wave);
    load.fetch(to + TILE, vh, row0, all.hi, wave);
  };
  typename TL::Lane at(smem + TL::bytes(ks * 32 * SUB), lane);
  if (NBUF == 2 && tiles > 0) fetch(smem, all.lo);   // in flight while delta is formed
  float delta = 0.f, largest = 0.f;
  {
    typename M::vec of[TL::FRAGS];
    if constexpr (LINES) {
      const unsigned rows = smem + 2 * TILE + wave * TL::bytes(32);
      load_frags_by_lines<E, D>(qf, rows, (const E*)a.q + h * dd, a.ldq, w0, a.T, lane, dd);
      load_frags_by_lines<E, D>(dof, rows, (const E*)a.dout + h * dd, a.ldo, w0, a.T, lane, dd);
      load_frags_by_lines<E, D>(of, rows, (const E*)a.o + h * dd, a.ldo, w0, a.T, lane, dd);
    } else TL::load_frags(of, (const E*)a.o + h * dd, a.ldo, my_q, a.T, lane, dd);
#pragma unroll
    for (int c = 0; c < TL::FRAGS; ++c)
#pragma unroll
      for (int e = 0; e < TL::VN; ++e) {
        delta = fmaf((float)dof[c][e], (float)of[c][e], delta);
        if constexpr (HALF<E>) largest = fmaxf(largest, fabsf((float)dof[c][e]));
      }
    delta += __shfl_xor(delta, 32, 64);
    if constexpr (HALF<E>) largest = fmaxf(largest, __shfl_xor(largest, 32, 64));
    if (ks == 0 && lane < 32 && my_q < a.T) {
      a.delta[stat] = delta;
      if constexpr (HALF<E>) a.delta[(int64_t)a.nh * a.T + stat] = largest;
    }
  }
  const float unit = HALF<E> ? unit_of(largest) : 1.f;
  f32x16 acc[TL::BLOCKS];
#pragma unroll
  for (int i = 0; i < TL::BLOCKS; ++i) acc[i] = f32x16{};
  if (NBUF == 2) {   // the second buffer's rows have been read, too
    tile_wait();
    __syncthreads();
  }
  for (int t = 0; t < tiles; ++t) {
    const int key0 = all.lo + t * ROWS;
    if (NBUF == 1) {
      fetch(smem, key0);
      tile_wait();
      __syncthreads();
    } else if (t + 1 < tiles) fetch(smem + ((t + 1) & 1) * 2 * TILE, key0 + ROWS);   // that buffer was last read before the barrier that ended the iteration before
    const int kb0 = key0 + ks * 32 * SUB;
    if (kb0 < mine.hi && kb0 + 32 * SUB > mine.lo) {
      const bool part = kb0 < mine.all_lo || kb0 + 32 * SUB > mine.all_hi;
#pragma unroll
      for (int j = 0; j < SUB; ++j) {
        const int kb = kb0 + 32 * j;
        f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
        for (int c = 0; c < TL::FRAGS; ++c) {
          s = M::rows(at.frag(0, 32 * j, c), qf[c], s);
          dp = M::rows(at.frag(TILE, 32 * j, c), dof[c], dp);
        }
        doc_weights<E, MODE>(s, dp, sc, (float)(kb + 4 * (lane >> 5) - my_q), DOC_UNIT<E, MODE> * unit, [&](int) { return f32x4{lse2, lse2, lse2, lse2}; },
                             [&](int) { return f32x4{delta, delta, delta, delta}; });
        if (part) {
          const int from = kb + 4 * (lane >> 5) - lo;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((unsigned)(from + 8 * (r >> 2) + (r & 3)) >= (unsigned)seen) dp[r] = 0.f;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const typename M::col8 df = pack<E>(dp, u);
#pragma unroll
          for (int b = 0; b < TL::BLOCKS; ++b) acc[b] = M::cols(at.column(0, 32 * j + 16 * u, b), df, acc[b]);
        }
      }
    }
    if (NBUF == 2) {
      tile_wait();
      at.move(t & 1 ? -2 * TILE : 2 * TILE);
    }
    __syncthreads();
  }
  if constexpr (KS > 1) merge_waves<TL::BLOCKS>(acc, reinterpret_cast<f32x4*>(smem_raw) + grp * (KS - 1) * TL::BLOCKS * 4 * 64, ks, KS, lane);
  DocRedo<NW>& redo = *reinterpret_cast<DocRedo<NW>*>(smem_raw);
  const unsigned again = redo_rows<NW>(redo, grp, ks == 0, ks == 0 && live && !(mark_of(acc) == 0.f));
  if (ks == 0) {
    if (!live) {
#pragma unroll
      for (int i = 0; i < TL::BLOCKS; ++i) acc[i] = f32x16{};
    }
    TL::store(acc, DOC_SLOPE<E, MODE> * a.scale / unit, smem_raw + (sizeof(redo) + 15) / 16 * 16 + grp * TL::STORE, (E*)a.dq + h * dd, a.lddq, w0, a.T,
              lane, dd, again);
  }
  if (__builtin_expect(any_row(redo.masks, GROUPS, lane), 0))   // the rows' delta: written by this workgroup, before its barrier
    redo_dq<E, NW>(&redo, GROUPS, row_groups, t0, a.ranges, a.T, dd, (const E*)a.q + blk.h * dd, a.ldq, kh, vh, a.ldkv, (const E*)a.dout + blk.h * dd, a.ldo,
                   a.lse + (int64_t)blk.h * a.T, a.delta + (int64_t)blk.h * a.T, a.scale, a.softcap, a.slopes ? a.slopes + blk.h : nullptr,
                   (E*)a.dq + blk.h * dd, a.lddq);
}

template <typename E, int D, int MODE, int NW, int KS, int ROWS>
__global__ __launch_bounds__(64 * NW, sizeof(E) == 2 && (NW == 8 || KS == 1) ? 2 : 1) void doc_dq_kernel(DocAttn a, int heads) {
  __shared__ __align__(16) char smem[dq_lds<E, D, NW, KS, ROWS, 2>()];
  dq_block<E, D, MODE, NW, KS, ROWS, 2>(smem, a, blockIdx.x, heads);
}

// ------------------------------------------------------------------------------------------ dK, dV
// dV^T += dO^T P, dK^T += Q^T dS with S = Q K^T: lanes are keys, registers rows. KG groups of 32 keys, each with QS waves, which share out the rows
// of a tile; a wave's V rows sit in LDS, which leaves registers for two waves per SIMD: all of them in heads of 128, where half spills up to 12, and
// bf16 with cap and bias 4 (in one launch with dQ up to 20 and 17). Bound like the forward, with 32 matrix instructions per block: 4096 tokens, 32
// heads, one document 275 us (1000 TFLOP/s of the 4 products), capped 308; dQ, with 24, 204 (1010 of 3) and 238.
template <typename E, int NW>
__device__ __attribute__((noinline)) void redo_dkv(DocRedo<NW>* redo, int groups, int t0, const int32_t* ranges, int T, int d, int group, const E* q,
                                                   int64_t ldq, const E* k, const E* v, int64_t ldkv, const E* dout, const E* o, int64_t ldo,
                                                   const float* lse, const float* delta, float scale, float softcap, const float* slopes, E* dk, E* dv, int64_t lddkv,
                                                   float* part_k, float* part_v, int64_t ld_part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for_dealt_rows(redo->masks, groups, NW, wave, [&](int g, int r) {
    const int j = t0 + 32 * g + r;
    const int4 range = doc_range((const int4*)ranges, j, T);
    wave_lds_order();
    row_to_lds(redo->rows[wave], k + j * ldkv, d, lane);
    row_to_lds(redo->rows[wave] + 128, v + j * ldkv, d, lane);
    wave_lds_order();
    float xk[2] = {0.f, 0.f}, xv[2] = {0.f, 0.f};
    for (int h = 0; h < group && !(all_nan(xk, d, lane) && all_nan(xv, d, lane)); ++h)
      doc_dkv_head<E>(redo->rows[wave], j, range.z, range.w, d, DocRows<E>{q + h * d, ldq}, DocRows<E>{dout + h * d, ldo}, DocRows<E>{o + h * d, ldo},
                      lse + (int64_t)h * T, delta ? delta + (int64_t)h * T : nullptr, scale, DocScore{softcap, slopes ? slopes[h] : 0.f}, lane, xk, xv);
#pragma unroll
    for (int c = 0; c < 2; ++c)
      if (64 * c + lane < d) {
        if (part_k) {
          part_k[j * ld_part + 64 * c + lane] = xk[c] * scale;
          part_v[j * ld_part + 64 * c + lane] = xv[c];
        } else {
          dk[j * lddkv + 64 * c + lane] = from_f<E>(xk[c] * scale);
          dv[j * lddkv + 64 * c + lane] = from_f<E>(xv[c]);
        }
      }
  });
}

template <typename E, int D, int KG, int QS, int ROWS, int NBUF> struct DkvLds {   // [NBUF][Q | dO], [NBUF][stats], [KG][V rows]
  typedef Tile<E, D> TL;
  static constexpr int STATS = HALF<E> ? 3 : 2, STAT = STATS * ROWS * 4;   // log-sum-exp in powers of two less P_SHIFT and g, delta, (half) largest |dO|
  static constexpr int V = NBUF * (2 * TL::bytes(ROWS) + STAT);
  static constexpr size_t LOOP = V + KG * TL::bytes(32), END = sizeof(DocRedo<KG * QS>) + 16 + KG * Tile<float, D>::STORE,
                          MERGE = (size_t)(QS - 1) * KG * TL::BLOCKS * 4 * 64 * 16;
  static constexpr size_t bytes = LOOP > END ? (LOOP > MERGE ? LOOP : MERGE) : END > MERGE ? END : MERGE;
};
// OWN: delta is formed here, from dO and the rows of o, by the wave that works on a row, instead of read.
template <typename E, int D, int MODE, int KG, int QS, int ROWS, int NBUF, bool OWN>
__device__ __forceinline__ void dkv_block(char* smem_raw, const DocAttn& a, int workgroup) {
  typedef Tile<E, D> TL;
  typedef Mat<E> M;
  typedef DkvLds<E, D, KG, QS, ROWS, NBUF> L;
  constexpr int NW = KG * QS, SUB = ROWS / 32 / QS, TILE = TL::bytes(ROWS), STATS = L::STATS, STAT = L::STAT, V = L::V;
  static_assert(ROWS <= 64 * NW && (!OWN || (KG == 1 && SUB == 1)), "");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qs = wave / KG, kg = wave % KG, dd = a.d, group = a.nh / a.nkv / a.parts;
  const int set = workgroup % (a.nkv * a.parts), kv = set % a.nkv, which = set / a.nkv, h0 = kv * (a.nh / a.nkv) + which * group;
  const int rank = workgroup / (a.nkv * a.parts);
  const int t0 = 32 * KG * (a.sorted ? heavy_block<true>(a.ranges, a.T, 32 * KG, (a.T + 32 * KG - 1) / (32 * KG), rank, lane) : rank);   // the longest first, in a document the early ones
  const int w0 = t0 + 32 * kg, my_k = w0 + (lane & 31);
  const E *kh = (const E*)a.k + kv * dd, *vh = (const E*)a.v + kv * dd;
  const unsigned smem = lds_address(smem_raw);
  const Span all = block_span<true, (32 * KG + 63) / 64>(a.ranges, t0, 32 * KG, a.T, lane);
  const int4 range = my_k < a.T ? doc_range((const int4*)a.ranges, my_k, a.T) : make_int4(0, 0, 0, 0);
  const int lo = range.z, seen = max(range.w - range.z, 0);
  typename M::vec kf[TL::FRAGS];
  constexpr bool LINES = ROWS >= 16 * KG;
  const unsigned k_at = smem + (NBUF - 1) * 2 * TILE + kg * TL::bytes(32);   // k comes by whole lines through the last buffer, where that holds the rows
  if constexpr (!LINES) TL::load_frags(kf, kh, a.ldkv, my_k, a.T, lane, dd);
  const Span mine = span_of(range.z, range.w);
  const int tiles = (all.hi - all.lo + ROWS - 1) / ROWS, total = tiles * group;
  if (qs == 0) {
    const TileLoad<E, D, 32, 1> load(a.ldkv, lane, dd);
    load.fetch(smem + V + kg * TL::bytes(32), vh, w0, a.T, 0);
    if constexpr (LINES) load.fetch(k_at, kh, w0, a.T, 0);
  }
  const TileLoad<E, D, ROWS, NW> load_q(a.ldq, lane, dd), load_d(a.ldo, lane, dd);
  float sr[STATS];
  typename M::vec of[OWN ? TL::FRAGS : 1];
  auto fetch = [&](int buf, int h, int row0) {
    if constexpr (OWN) TL::load_frags(of, (const E*)a.o + h * dd, a.ldo, row0 + 32 * qs + (lane & 31), a.T, lane, dd);
    load_q.fetch(smem + buf * 2 * TILE, (const E*)a.q + h * dd, row0, all.hi, wave);
    load_d.fetch(smem + buf * 2 * TILE + TILE, (const E*)a.dout + h * dd, row0, all.hi, wave);
    if (tid < ROWS) {
      const int64_t from = (int64_t)h * a.T + min(row0 + tid, a.T - 1);
      sr[0] = a.lse[from];
      if constexpr (!OWN) sr[1] = a.delta[from];
      if constexpr (HALF<E> && !OWN) sr[2] = a.delta[(int64_t)a.nh * a.T + from];
    }
  };
  DocScale sc = doc_scale<E, MODE>(a, h0);
  const float minus = P_SHIFT<E> + sc.g;
  auto put_stats = [&](int buf, int row0) {
    float* st = reinterpret_cast<float*>(smem_raw + NBUF * 2 * TILE + buf * STAT);
    if (tid < ROWS) {   // rows past the end: zeros, whose weights 1 meet rows of zeros
      const bool in = row0 + tid < all.hi;
      st[tid] = in ? fmaf(sr[0], DOC_LOG2E, -minus) : 0.f;
      if constexpr (!OWN) st[ROWS + tid] = in ? sr[1] : 0.f;
      if constexpr (HALF<E> && !OWN) st[2 * ROWS + tid] = in ? sr[2] : 0.f;
    }
  };
  f32x16 dk[TL::BLOCKS], dv[TL::BLOCKS];
#pragma unroll
  for (int i = 0; i < TL::BLOCKS; ++i) dk[i] = dv[i] = f32x16{};
  float unit = 0.f;   // half: of the lane's score gradients, none yet
  int h = h0, t = 0;
  if (NBUF == 2 && total > 0) {
    fetch(0, h, all.lo);
    put_stats(0, all.lo);
  }
  tile_wait();
  __syncthreads();
  if constexpr (LINES) {
    const typename TL::Lane at_k(k_at, lane);
#pragma unroll
    for (int s = 0; s < TL::FRAGS; ++s) kf[s] = at_k.frag(0, 0, s);
    __syncthreads();   // before that buffer's first tile
  }
  typename TL::Lane at(smem + TL::bytes(qs * 32 * SUB), lane);
  const typename TL::Lane at_v(smem + V + kg * TL::bytes(32), lane);
  unsigned stat_at = smem + NBUF * 2 * TILE + 4 * (qs * 32 * SUB + 4 * (lane >> 5));
  for (int it = 0; it < total; ++it) {
    const int row0 = all.lo + t * ROWS, buf = NBUF == 2 ? it & 1 : 0;
    const int tn = t + 1 < tiles ? t + 1 : 0, hn = tn ? h : h + 1, rown = all.lo + tn * ROWS;
    if (NBUF == 1) {
      fetch(0, h, row0);
      put_stats(0, row0);
      tile_wait();
      __syncthreads();
    }
    if constexpr (OWN) {   // lane and lane ^ 32 hold a row
      float x = 0.f, largest = 0.f;
#pragma unroll
      for (int c = 0; c < TL::FRAGS; ++c) {
        const typename M::vec d = at.frag(TILE, 0, c);
#pragma unroll
        for (int e = 0; e < TL::VN; ++e) {
          x = fmaf((float)d[e], (float)of[c][e], x);
          if constexpr (HALF<E>) largest = fmaxf(largest, fabsf((float)d[e]));
        }
      }
      x += __shfl_xor(x, 32, 64);
      const unsigned to = stat_at - 16 * (lane >> 5) + 4 * (lane & 31);
      *(__attribute__((address_space(3))) float*)(uintptr_t)(to + 4 * ROWS) = x;
      if constexpr (HALF<E>) *(__attribute__((address_space(3))) float*)(uintptr_t)(to + 8 * ROWS) = fmaxf(largest, __shfl_xor(largest, 32, 64));
      wave_lds_order();
    }
    if (NBUF == 2 && it + 1 < total) fetch(buf ^ 1, hn, rown);
    const int rb0 = row0 + qs * 32 * SUB;
    if (rb0 < mine.hi && rb0 + 32 * SUB > mine.lo) {
      const bool part = rb0 < mine.all_lo || rb0 + 32 * SUB > mine.all_hi;
#pragma unroll
      for (int j = 0; j < SUB; ++j) {
        const int rb = rb0 + 32 * j;
        if constexpr (HALF<E>) {   // the unit of a key, and lane, follows the largest |dO| of the rows so far that see it
          float top = 0.f;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            f32x4 x = lds_read<f32x4>(stat_at + 4 * (2 * ROWS + 32 * j + 8 * c));
            if (part) {
              const int from = rb + 4 * (lane >> 5) - lo;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if ((unsigned)(from + 8 * c + e) >= (unsigned)seen) x[e] = 0.f;
            }
            top = fmaxf(top, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
          }
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float now = unit_of(top);
          const bool moves = top > 0.f && (unit == 0.f || now < unit);
          if (__any(moves)) {
            const float f = moves && unit != 0.f ? now / unit : 1.f;
            if (moves) unit = now;
#pragma unroll
            for (int b = 0; b < TL::BLOCKS; ++b)
#pragma unroll
              for (int r = 0; r < 16; ++r) dk[b][r] *= f;
          }
          __builtin_amdgcn_sched_barrier(0);   // before the products: behind them heads of 128 spill 100 registers (backward of 4096 tokens 214 -> 445 us)
        }
        f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
        for (int c = 0; c < TL::FRAGS; ++c) {
          s = M::rows(at.frag(0, 32 * j, c), kf[c], s);
          dp = M::rows(at.frag(TILE, 32 * j, c), at_v.frag(0, 0, c), dp);
        }
        // Two waves per SIMD have 256 registers each, of which 192 hold K, dK, dV and the scores: the phases are kept apart, or the compiler
        // spills accumulators to read ahead.
        if constexpr (sizeof(E) == 2) __builtin_amdgcn_sched_barrier(0);
        doc_weights<E, MODE>(s, dp, sc, (float)(rb + 4 * (lane >> 5) - my_k), HALF<E> ? DOC_UNIT<E, MODE> / 16384.f * unit : 1.f,
                             [&](int c) { return lds_read<f32x4>(stat_at + 4 * (32 * j + 8 * c)); },
                             [&](int c) { return lds_read<f32x4>(stat_at + 4 * (ROWS + 32 * j + 8 * c)); });
        if (part) {
          const int from = rb + 4 * (lane >> 5) - lo;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((unsigned)(from + 8 * (r >> 2) + (r & 3)) >= (unsigned)seen) s[r] = dp[r] = 0.f;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if constexpr (sizeof(E) == 2) __builtin_amdgcn_sched_barrier(0);
          const typename M::col8 pf = pack<E>(s, u), df = pack<E>(dp, u);
#pragma unroll
          for (int b = 0; b < TL::BLOCKS; ++b) {
            dv[b] = M::cols(at.column(TILE, 32 * j + 16 * u, b), pf, dv[b]);
            dk[b] = M::cols(at.column(0, 32 * j + 16 * u, b), df, dk[b]);
          }
        }
      }
    }
    if (NBUF == 2) {
      if (it + 1 < total) put_stats(buf ^ 1, rown);
      tile_wait();
      at.move(buf ? -2 * TILE : 2 * TILE);
      stat_at += buf ? -STAT : STAT;
    }
    __syncthreads();
    if (hn != h && it + 1 < total) sc = doc_scale<E, MODE>(a, hn);
    t = tn;
    h = hn;
  }
  if constexpr (HALF<E>) {
    if constexpr (QS > 1) {   // the waves that share keys bring theirs to the unit of 1 before they add
      const float f = unit == 0.f ? 1.f : 1.f / unit;
#pragma unroll
      for (int b = 0; b < TL::BLOCKS; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[b][r] *= f;
      unit = 1.f;
    }
  }
  if constexpr (QS > 1) {
    f32x4* red = reinterpret_cast<f32x4*>(smem_raw) + kg * (QS - 1) * TL::BLOCKS * 4 * 64;
    merge_waves<TL::BLOCKS>(dv, red, qs, QS, lane);
    merge_waves<TL::BLOCKS>(dk, red, qs, QS, lane);
  }
  const bool live = seen > 0 && my_k < a.T;
  const int64_t ld_part = a.nkv * dd;
  float *part_k = a.partial + (int64_t)which * a.T * ld_part + kv * dd, *part_v = part_k + (int64_t)a.parts * a.T * ld_part;
  DocRedo<NW>& redo = *reinterpret_cast<DocRedo<NW>*>(smem_raw);
  const unsigned again = redo_rows<NW>(redo, kg, qs == 0, qs == 0 && live && !(mark_of(dk) + mark_of(dv) == 0.f));
  if (qs == 0) {
    if (!live) {
#pragma unroll
      for (int i = 0; i < TL::BLOCKS; ++i) dk[i] = dv[i] = f32x16{};
    }
    char* to = smem_raw + (sizeof(redo) + 15) / 16 * 16 + kg * Tile<float, D>::STORE;
    const float fv = HALF<E> ? 1.f / 16384.f : 1.f, fk = DOC_SLOPE<E, MODE> * (HALF<E> && unit != 0.f ? a.scale / unit : a.scale);
    if (a.parts > 1) {
      Tile<float, D>::store(dv, fv, to, part_v, ld_part, w0, a.T, lane, dd, again);
      Tile<float, D>::store(dk, fk, to, part_k, ld_part, w0, a.T, lane, dd, again);
    } else {
      TL::store(dv, fv, to, (E*)a.dv + kv * dd, a.lddkv, w0, a.T, lane, dd, again);
      TL::store(dk, fk, to, (E*)a.dk + kv * dd, a.lddkv, w0, a.T, lane, dd, again);
    }
  }
  if (__builtin_expect(any_row(redo.masks, KG, lane), 0))
    redo_dkv<E, NW>(&redo, KG, t0, a.ranges, a.T, dd, group, (const E*)a.q + h0 * dd, a.ldq, kh, vh, a.ldkv, (const E*)a.dout + h0 * dd,
                    (const E*)a.o + h0 * dd, a.ldo, a.lse + (int64_t)h0 * a.T, OWN ? nullptr : a.delta + (int64_t)h0 * a.T, a.scale, a.softcap,
                    a.slopes ? a.slopes + h0 : nullptr, (E*)a.dk + kv * dd, (E*)a.dv + kv * dd, a.lddkv, a.parts > 1 ? part_k : nullptr, part_v, ld_part);
}

template <typename E, int D, int MODE, int KG, int QS, int ROWS, int NBUF>
__global__ __attribute__((amdgpu_waves_per_eu(sizeof(E) == 2 ? 2 : 1, sizeof(E) == 2 ? 2 : 1))) __launch_bounds__(64 * KG * QS) void doc_dkv_kernel(DocAttn a) {
  __shared__ __align__(16) char smem[DkvLds<E, D, KG, QS, ROWS, NBUF>::bytes];
  dkv_block<E, D, MODE, KG, QS, ROWS, NBUF, false>(smem, a, blockIdx.x);
}

// Both in one launch, for few rows, where one after the other would leave most of the chip idle twice: no block reads what another one writes.  One buffer
// where two workgroups then fit a CU, whose waits overlap (fp32 heads over 64: one workgroup in any case).  us, one after the other : together: 256
// tokens, 4 heads of 128, bf16 24.4 : 16.7; 500 tokens, 8 heads 29.4 : 23.0; fp32, 1000 tokens, 8 heads of 64 over 2 74.5 : 53.2.
template <typename E, int D> constexpr int FEW_BUFFERS = sizeof(E) == 2 && D == 64 ? 2 : 1;
template <typename E, int D> constexpr int FEW_WAVES = sizeof(E) == 4 && D > 64 ? 1 : 2;   // per SIMD
template <typename E, int D, int MODE>
__global__ __attribute__((amdgpu_waves_per_eu(FEW_WAVES<E, D>, FEW_WAVES<E, D>))) __launch_bounds__(256) void doc_bwd_kernel(DocAttn a, int dkv_workgroups) {
  constexpr int N = FEW_BUFFERS<E, D>;
  constexpr size_t A = DkvLds<E, D, 1, 4, 128, N>::bytes, B = dq_lds<E, D, 4, 4, 128, N>();
  __shared__ __align__(16) char smem[A > B ? A : B];
  if ((int)blockIdx.x < dkv_workgroups) dkv_block<E, D, MODE, 1, 4, 128, N, true>(smem, a, blockIdx.x);
  else dq_block<E, D, MODE, 4, 4, 128, N>(smem, a, blockIdx.x - dkv_workgroups, 1);
}

// Where the query heads of a key head are shared out over `parts` workgroups, these leave their sums in fp32; they meet here, in the order of the parts.
template <typename E> __global__ __launch_bounds__(256) void doc_join_kernel(DocAttn a) {
  constexpr int VN = 16 / sizeof(E);
  typedef typename Vec<E>::type vec;
  const int row = a.nkv * a.d / VN;   // vectors of a token
  const int64_t n = (int64_t)a.T * row, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= 2 * n) return;
  const bool is_v = at >= n;
  const int64_t i = is_v ? at - n : at, t = i / row;
  const int c = (int)(i - t * row) * VN;
  float sum[VN] = {};
  for (int p = 0; p < a.parts; ++p) {
    const float* from = a.partial + (((int64_t)(is_v ? a.parts : 0) + p) * a.T + t) * (a.nkv * a.d) + c;
#pragma unroll
    for (int e = 0; e < VN; e += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(from + e);
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[e + k] += x[k];
    }
  }
  vec o;
#pragma unroll
  for (int e = 0; e < VN; ++e) o[e] = from_f<E>(sum[e]);
  *reinterpret_cast<vec*>((E*)(is_v ? a.dv : a.dk) + t * a.lddkv + c) = o;
}

// Heads of a key head that share a workgroup of `groups` waves.
inline int doc_heads(const DocAttn& a, int groups) {
  const int group = a.nh / a.nkv;
  return groups % 4 == 0 && group % 4 == 0 ? 4 : groups % 2 == 0 && group % 2 == 0 ? 2 : 1;
}
// The longest blocks first by their ranges: where the workgroups are more than the chip holds at a time, and the blocks few enough to be ordered (six
// documents in 4096 tokens: forward 74 -> 66 us, dQ 107 -> 98, dK/dV 160 -> 144).
inline bool doc_sorted(int64_t blocks, int64_t workgroups, int per_cu) { return blocks <= 256 && workgroups > 256 * per_cu; }

// Waves that share rows, and rows of the tiles that they share out, as far as two buffers fit in LDS.
template <typename E, int D> constexpr int SHARE = sizeof(E) == 4 && D > 64 ? 2 : 4;
template <typename E, int D, int MODE, int NW, int KS, int ROWS, bool BWD> hipError_t doc_rows(hipStream_t st, DocAttn a) {
  const int heads = doc_heads(a, NW / KS);
  const int64_t blocks = cdiv(a.T, 32 * (NW / KS) / heads), wgs = blocks * (a.nh / heads);
  a.sorted = doc_sorted(blocks, wgs, NW == 4 && KS == 1 ? 2 : 1);
  if constexpr (BWD) hipLaunchKernelGGL((doc_dq_kernel<E, D, MODE, NW, KS, ROWS>), dim3((unsigned)wgs), dim3(64 * NW), 0, st, a, heads);
  else hipLaunchKernelGGL((doc_fwd_kernel<E, D, MODE, NW, KS, ROWS>), dim3((unsigned)wgs), dim3(64 * NW), 0, st, a, heads);
  return hipGetLastError();
}
// The forward's and dQ's workgroups by the groups of 32 rows that there are, for 1024 SIMDs: with few of them the waves of a workgroup share rows and
// each walks a part of the keys. us, bf16, heads of 128, one document (in brackets three of 48, 34 and 15 %), heads of 64 alike:
//   256 groups, four waves on 32 rows : eight on 64.  2048 tokens 24.9 : 23.9 (16.0 : 16.1); 1024 tokens 192 groups 16.2 : 15.9, 384 groups 22.1 : 16.1
//   768 groups, eight waves on 64 rows : on 128.  512 groups, 1024 tokens 17.5 : 20.7 (12.3 : 13.6), 2048 tokens 24.6 : 32.0 (16.8 : 19.8); 640 groups
//     22.0 : 20.8 (19.4 : 14.5) and 30.6 : 35.1 (22.2 : 21.8); 768 groups 23.6 : 20.3 (20.4 : 13.9) and 30.8 : 33.9 (23.3 : 21.2); longer documents
//     alone would have the cut later, packed ones earlier
//   2048 groups, eight waves on 128 rows : four.  Two eight-wave workgroups for every CU, one after the other; more begin a third turn. 2048 tokens,
//     1792 groups 45.8 : 47.5 (31.6 : 32.2), 2048 groups 48.6 : 49.9 (33.3 : 31.5), 2560 groups 66.9 : 55.1 (45.1 : 34.4); 4096 tokens, 1536 groups
//     68.3 : 82.0 (37.5 : 51.9), 2048 groups 79.9 : 90.6 (46.7 : 49.8), 4096 groups 156 : 152 (86.9 : 68.5)
// dQ likewise. Eight waves on 256 rows: 4096 tokens, 32 heads over 8, six documents 84, four on 128 rows 75, one document 144 and 155: the only kind
// that gains, by 7 % and less the longer.
template <typename E, int D, int MODE, bool BWD> hipError_t doc_by_rows(hipStream_t st, const DocAttn& a) {
  constexpr int S = SHARE<E, D>;
  const int64_t groups = cdiv(a.T, 32) * a.nh;
  if constexpr (!BWD)   // the backward of so few rows takes doc_bwd_kernel
    if (groups < (sizeof(E) == 2 ? 256 : 1024)) return doc_rows<E, D, MODE, 4, S, 32 * S, BWD>(st, a);
  if constexpr (sizeof(E) == 2) {
    if (groups < 768) return doc_rows<E, D, MODE, 8, 4, 128, BWD>(st, a);
    if (groups <= 2048) return doc_rows<E, D, MODE, 8, 2, 128, BWD>(st, a);
    return doc_rows<E, D, MODE, 4, 1, 64, BWD>(st, a);
  } else return doc_rows<E, D, MODE, 4, 1, 32, BWD>(st, a);
}
template <typename E> hipError_t doc_join(hipStream_t st, const DocAttn& a) {
  if (a.parts > 1) hipLaunchKernelGGL(doc_join_kernel<E>, dim3((unsigned)cdiv(2 * (int64_t)a.T * (a.nkv * a.d / (16 / (int)sizeof(E))), 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <typename E, int D, int MODE, int KG, int QS, int ROWS, int NBUF> hipError_t doc_dkv(hipStream_t st, DocAttn a) {
  const int64_t blocks = cdiv(a.T, 32 * KG), wgs = blocks * a.nkv * a.parts;
  a.sorted = doc_sorted(blocks, wgs, sizeof(E) == 2 && KG * QS == 4 ? 2 : 1);
  hipLaunchKernelGGL((doc_dkv_kernel<E, D, MODE, KG, QS, ROWS, NBUF>), dim3((unsigned)wgs), dim3(64 * KG * QS), 0, st, a);
  return hipGetLastError();
}
// dK/dV's workgroups: with many key blocks, four waves on 128 keys, two workgroups to a CU, which hide one another's beginnings and ends; with fewer
// four waves on 64 keys; below that eight waves on 64 keys, and then the query heads of a key head in parts (doc_dkv_parts); with few rows one launch
// with dQ. us of the whole backward, bf16, heads of 128, one document (in brackets three of 48, 34 and 15 %), heads of 64 alike but for the first
// cut, which they would have at twice the rows:
//   256 blocks of 64 keys and query head, one launch : eight waves.  2048 tokens, 8 heads (256) 68 : 66 (44.8 : 45.7); 1024 tokens, 12 heads (192) 40.4
//     : 41.8 (30.0 : 32.5), 16 heads (256) 46.6 : 42.9 (35.7 : 32.8), 20 heads 58.3 : 54.7 (42.9 : 48.5)
//   384 blocks of 128 keys, eight waves : four, 64 keys.  2048 tokens, 320 blocks 120 : 116 (79 : 73), 384 130 : 117 (87 : 74); 4096 tokens, 320 blocks
//     205 : 216 (112 : 117), 384 223 : 225 (119 : 121), 448 252 : 247 (141 : 132)
//   1024 blocks of 128 keys, four, 64 keys : 128 keys.  2048 tokens, 768 blocks 216 : 204 (125 : 118), 1024 283 : 263 (162 : 145); 4096 tokens, 768 385
//     : 376 (182 : 187), 1024 504 : 483 (234 : 219), 1280 620 : 593 (298 : 281)
// 8 key heads, 4096 tokens, capped, in two parts 236 and 216, whole 207. Eight waves on 128 keys, which bring in half the rows, are never the
// fastest: 190, 178, 275 where four on 128, four on 64 and eight on 64 take 175, 168 and 207.
template <typename E, int D, int MODE> hipError_t doc_bwd(hipStream_t st, const DocAttn& a) {
  const int keys = doc_dkv_keys((DType)(sizeof(E) == 4 ? F32 : BF16), a.T, a.nh, a.nkv);
  if (keys == 32) {
    const int64_t dkv = cdiv(a.T, 32) * a.nkv * a.parts, dq = cdiv(a.T, 32) * a.nh;
    hipLaunchKernelGGL((doc_bwd_kernel<E, D, MODE>), dim3((unsigned)(dkv + dq)), dim3(256), 0, st, a, (int)dkv);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : doc_join<E>(st, a);
  }
  hipError_t e = doc_by_rows<E, D, MODE, true>(st, a);
  if (e != hipSuccess) return e;
  if constexpr (sizeof(E) == 4) e = doc_dkv<E, D, MODE, 4, 1, 32, 2>(st, a);
  else if (keys == 128) e = doc_dkv<E, D, MODE, 4, 1, 32, 2>(st, a);
  else if (cdiv(a.T, 128) * a.nkv >= 384) e = doc_dkv<E, D, MODE, 2, 2, 64, 1>(st, a);
  else e = doc_dkv<E, D, MODE, 2, 4, 128, 2>(st, a);
  return e != hipSuccess ? e : doc_join<E>(st, a);
}
template <typename E, int D, int MODE> hipError_t doc_either(hipStream_t st, const DocAttn& a, bool backward) {
  return backward ? doc_bwd<E, D, MODE>(st, a) : doc_by_rows<E, D, MODE, false>(st, a);
}
template <typename E, int D> hipError_t doc_mode(hipStream_t st, const DocAttn& a, bool backward) {
  const bool cap = a.softcap > 0.f;
  return cap ? (a.slopes ? doc_either<E, D, DOC_CAP | DOC_BIAS>(st, a, backward) : doc_either<E, D, DOC_CAP>(st, a, backward))
             : (a.slopes ? doc_either<E, D, DOC_BIAS>(st, a, backward) : doc_either<E, D, DOC_PLAIN>(st, a, backward));
}

}  // namespace

// Heads are padded with zeros to D = 64, 96 or 128.
template <typename E> hipError_t doc_attention(hipStream_t st, const DocAttn& a, bool backward) {
  return a.d <= 64 ? doc_mode<E, 64>(st, a, backward) : a.d <= 96 ? doc_mode<E, 96>(st, a, backward) : doc_mode<E, 128>(st, a, backward);
}

}  // namespace zs
