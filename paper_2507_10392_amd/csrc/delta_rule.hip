// The gated delta rule: the table of a microbatch's chunks, the choice of the element type's kernels (delta_rule_impl.h), and single tokens.
#include "kernels.h"

#include <algorithm>

namespace zs {

hipError_t delta_rule_bf16(hipStream_t st, const DeltaRule& a, bool backward);
hipError_t delta_rule_f16(hipStream_t st, const DeltaRule& a, bool backward);
hipError_t delta_rule_f32(hipStream_t st, const DeltaRule& a, bool backward);

namespace {

// ------------------------------------------------------------------------------------------ chunks
// One workgroup.  Whatever the offsets hold, documents are clipped to [0, T] and to the chunks that the table has room for (delta_table.h), so that no row
// of the table leads outside, and none is written outside of the table.  Rows of documents come longest first where there are at most SORTED (the walks from
// chunk to chunk take as long as the longest), those of more as they are.  Layout, rows of four: (0, first and end of the documents' tokens, 0); per document
// (first token, tokens, first chunk, document); per chunk (first token, tokens or 0: no chunk, document, place in it).
// Bound by steps that follow one another, of which every wave has one per document for the rows of its chunks: 11.4 us for up to 64 documents, 53 for 1024 of 64
// tokens (more than half of it their order), 3 ms for 2^18.  Once a microbatch, for all layers and both directions, so one workgroup was left to do it.
constexpr int TABLE_THREADS = DELTA_TURN, SORTED = DELTA_TURN;
__global__ __launch_bounds__(TABLE_THREADS) void delta_chunks_kernel(int T, int ndocs, int nchunks, const int32_t* __restrict__ offsets, int4* __restrict__ table) {
  __shared__ int waves[TABLE_THREADS / 64], lengths[SORTED];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int4 *docs = table + 1, *chunks = docs + ndocs;
  if (tid == 0) {
    const int begin = min(max(offsets[0], 0), T);
    table[0] = make_int4(0, begin, min(max(offsets[ndocs], begin), T), 0);
  }
  int before = 0;   // chunks of the documents of earlier turns, nchunks at most
  for (int d0 = 0; d0 < ndocs; d0 += TABLE_THREADS) {
    const int d = d0 + tid;
    int first = 0, count = 0;
    if (d < ndocs) {
      first = min(max(offsets[d], 0), T);
      count = max(min(max(offsets[d + 1], 0), T) - first, 0);
    }
    const int mine = delta_chunks_of(count);
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum, o, 64);
      if (lane >= o) sum += x;
    }
    if (lane == 63) waves[wave] = sum;
    if (ndocs <= SORTED && d < ndocs) lengths[d] = count;
    __syncthreads();
    int base = 0, turn = 0;
    for (int w = 0; w < TABLE_THREADS / 64; ++w) {
      if (w < wave) base += waves[w];
      turn += waves[w];
    }
    const DeltaPlace at = delta_place(before, base + sum - mine, count, nchunks);
    const int chunk0 = at.chunk0;
    count = at.tokens;
    before = delta_turn_end(before, turn, nchunks);
    if (d < ndocs) {
      int place = d;
      if (ndocs <= SORTED) {
        place = 0;
        const int own = lengths[d];
        for (int o = 0; o < ndocs; ++o) place += lengths[o] > own || (lengths[o] == own && o < d);
      }
      docs[place] = make_int4(first, count, chunk0, d);
    }
    // the wave's documents' chunks, a document after the other
    for (int l = 0; l < 64; ++l) {
      const int f = __shfl(first, l, 64), n = __shfl(count, l, 64), c0 = __shfl(chunk0, l, 64);
      for (int i = lane; i < delta_chunks_of(n); i += 64)
        chunks[c0 + i] = make_int4(f + DELTA_CHUNK * i, min(n - DELTA_CHUNK * i, DELTA_CHUNK), d0 + 64 * wave + l, i);
    }
    __syncthreads();
  }
  for (int c = before + tid; c < nchunks; c += TABLE_THREADS) chunks[c] = make_int4(0, 0, 0, 0);
}

// ------------------------------------------------------------------------------------------ single tokens
// Memory bound: a state is read and written once.  A workgroup has 32 columns of a state, whole 128-byte lines of its rows, which are independent of
// the others: with w = a S, r = w^T k, t = w^T q (both sums over the rows, in one pass), u = beta (v - r), S = w + k u^T, o = scale (t + (q.k) u).
// Tokens of one state in one call come in their order: the workgroup of the first takes them all.  bf16, 32 heads of 128: 48 tokens 35 us, 203 MB at 5.8 TB/s; one
// 5.3, the latencies of a slot, its state and the store.  Splitting a state further, by rows, would need a second launch for the sums.
constexpr int STEP_ROWS = 4;   // of a thread, at most: 128 rows by 32 groups of eight threads
template <typename E> __global__ __launch_bounds__(256) void delta_step_kernel(DeltaStep a) {
  __shared__ float qs[128], ks[128], sums[4][2][32], red[4];
  __shared__ int found[4][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, group = tid >> 3;
  const int slices = (a.dv + 31) / 32, h = (int)blockIdx.x / slices, col = (int)blockIdx.x % slices * 32 + (tid & 7) * 4;
  const int kv = h / (a.nv / a.nk);
  const bool live = col < a.dv;
  int token = blockIdx.y;
  const int slot = a.slots ? a.slots[token] : token;
  if (slot < 0 || slot >= a.nstates) {
    if (tid < 8 && live) {
      E* o = (E*)a.o + (int64_t)token * a.ldo + h * a.dv + col;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = from_f<E>(0.f);
    }
    return;
  }
  float* state = a.state + ((int64_t)slot * a.nv + h) * a.dk * a.dv + col;
  f32x4 w[STEP_ROWS];
#pragma unroll
  for (int i = 0; i < STEP_ROWS; ++i) {
    const int r = group + 32 * i;
    w[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (r < a.dk && live) w[i] = *reinterpret_cast<const f32x4*>(state + (int64_t)r * a.dv);
  }
  for (;;) {
    int next = a.n;
    if (a.slots) {   // an earlier token of this state takes it; else the next one behind this
      int before = 0;
      for (int j = tid; j < a.n; j += 256) {
        const bool same = a.slots[j] == slot;
        before |= same && j < token;
        if (same && j > token) next = min(next, j);
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) next = min(next, __shfl_xor(next, o, 64));
      before = __any(before);
      if (lane == 0) {
        found[wave][0] = before;
        found[wave][1] = next;
      }
    }
    const float decay = expf(a.g[(int64_t)token * a.nv + h]), beta = a.beta[(int64_t)token * a.nv + h];
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (live) {
      const E* from = (const E*)a.v + (int64_t)token * a.ldv + h * a.dv + col;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = to_f(from[e]);
    }
    if (tid < a.dk) {
      qs[tid] = to_f(((const E*)a.q)[(int64_t)token * a.ldq + kv * a.dk + tid]);
      ks[tid] = to_f(((const E*)a.k)[(int64_t)token * a.ldk + kv * a.dk + tid]);
    }
    __syncthreads();
    if (a.slots) {
      next = min(min(found[0][1], found[1][1]), min(found[2][1], found[3][1]));
      if (token == (int)blockIdx.y && (found[0][0] | found[1][0] | found[2][0] | found[3][0])) return;
    }
    f32x4 r = {0.f, 0.f, 0.f, 0.f}, t = r;
    float qk = tid < a.dk ? qs[tid] * ks[tid] : 0.f;
#pragma unroll
    for (int i = 0; i < STEP_ROWS; ++i) {
      const int row = group + 32 * i;
      w[i] *= decay;
      if (row < a.dk) {
        r += w[i] * ks[row];
        t += w[i] * qs[row];
      }
    }
#pragma unroll
    for (int o = 8; o < 64; o <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        r[e] += __shfl_xor(r[e], o, 64);
        t[e] += __shfl_xor(t[e], o, 64);
      }
    qk = wave_sum(qk);
    if (lane < 8) {
      *reinterpret_cast<f32x4*>(&sums[wave][0][4 * lane]) = r;
      *reinterpret_cast<f32x4*>(&sums[wave][1][4 * lane]) = t;
    }
    if (lane == 0) red[wave] = qk;
    __syncthreads();
    r = t = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r += *reinterpret_cast<const f32x4*>(&sums[i][0][4 * (tid & 7)]);
      t += *reinterpret_cast<const f32x4*>(&sums[i][1][4 * (tid & 7)]);
    }
    qk = (red[0] + red[1]) + (red[2] + red[3]);
    const f32x4 u = (v - r) * beta;   // (of columns that are not live: zeros, which nobody stores)
#pragma unroll
    for (int i = 0; i < STEP_ROWS; ++i) {
      const int row = group + 32 * i;
      if (row < a.dk) w[i] += u * ks[row];
    }
    if (tid < 8 && live) {
      E* o = (E*)a.o + (int64_t)token * a.ldo + h * a.dv + col;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = from_f<E>(fp32_value(a.scale * (t[e] + qk * u[e])));
    }
    if (next >= a.n) break;
    token = next;
    __syncthreads();   // the token before is done with the LDS
  }
#pragma unroll
  for (int i = 0; i < STEP_ROWS; ++i) {
    const int r = group + 32 * i;
    if (r < a.dk && live) *reinterpret_cast<f32x4*>(state + (int64_t)r * a.dv) = w[i];
  }
}

struct DeltaScratch { int64_t records, halves, states, dstates, u, y, total; };
DeltaScratch delta_layout(DType dt, bool backward, int T, int ndocs, int nk, int nv, int dk, int dv) {
  const int64_t chunks = delta_chunk_rows(T, ndocs), n = chunks * nv, rows = dk <= 64 ? 64 : 128, dvp = cdiv(dv, 16) * 16;
  DeltaScratch s = {};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t p = at;
    at += cdiv(bytes, 256) * 256;
    return p;
  };
  s.records = take(n * (backward ? DELTA_RECORD_BWD : DELTA_RECORD_FWD));
  s.halves = take(dt == BF16 ? chunks * nk * 2 * DELTA_CHUNK * rows * 2 : 0);   // bf16 keys and queries
  if (backward) {
    s.states = take(n * rows * dvp * 4);
    s.dstates = take(n * rows * dvp * 4);
    s.u = take(n * DELTA_CHUNK * dvp * 4);
    s.y = take(n * DELTA_CHUNK * dvp * 4);
  }
  s.total = std::max<int64_t>(at, 256);
  return s;
}
}  // namespace

int64_t delta_chunk_rows(int T, int ndocs) { return (int64_t)T / DELTA_CHUNK + std::min(T, ndocs); }
hipError_t delta_chunks(hipStream_t st, int T, int ndocs, const int32_t* offsets, int32_t* table) {
  hipLaunchKernelGGL(delta_chunks_kernel, dim3(1), dim3(TABLE_THREADS), 0, st, T, ndocs, (int)delta_chunk_rows(T, ndocs), offsets, (int4*)table);
  return hipGetLastError();
}
int64_t delta_scratch(DType dt, bool backward, int T, int ndocs, int nk, int nv, int dk, int dv) {
  return delta_layout(dt, backward, T, ndocs, nk, nv, dk, dv).total;
}
hipError_t delta_rule(hipStream_t st, DType dt, const DeltaRule& in, bool backward, void* scratch) {
  DeltaRule a = in;
  const DeltaScratch s = delta_layout(dt, backward, a.T, a.ndocs, a.nk, a.nv, a.dk, a.dv);
  char* base = (char*)scratch;
  a.nchunks = (int)delta_chunk_rows(a.T, a.ndocs);
  a.dvp = (int)(cdiv(a.dv, 16) * 16);
  a.records = base + s.records;
  a.halves = (f16*)(base + s.halves);
  a.states = (float*)(base + s.states);
  a.dstates = (float*)(base + s.dstates);
  a.u = (float*)(base + s.u);
  a.y = (float*)(base + s.y);
  return dt == F32 ? delta_rule_f32(st, a, backward) : dt == BF16 ? delta_rule_bf16(st, a, backward) : delta_rule_f16(st, a, backward);
}
hipError_t delta_step(hipStream_t st, DType dt, const DeltaStep& a) {
  const dim3 grid((unsigned)(a.nv * cdiv(a.dv, 32)), (unsigned)a.n), blk(256);
  if (dt == F32) hipLaunchKernelGGL(delta_step_kernel<float>, grid, blk, 0, st, a);
  else if (dt == BF16) hipLaunchKernelGGL(delta_step_kernel<bf16>, grid, blk, 0, st, a);
  else hipLaunchKernelGGL(delta_step_kernel<f16>, grid, blk, 0, st, a);
  return hipGetLastError();
}

}  // namespace zs
