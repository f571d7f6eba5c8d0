// What packed documents need besides attention: the ranges of keys and rows that see one another, and rotary positions with several
// axes.
#include "kernels.h"

namespace zs {
namespace {

// ------------------------------------------------------------------------------------------ ranges
// One thread per token finds its document by halving.  Whatever the offsets hold, the ranges stay inside [0, T): documents are
// clipped to it, and a token outside the document that the search ends at sees nothing.
__global__ __launch_bounds__(256) void doc_ranges_kernel(int T, int ndocs, const int32_t* __restrict__ offsets, const int32_t* __restrict__ prefix,
                                                         int4* __restrict__ ranges) {
  const int t = (int)(blockIdx.x * 256 + threadIdx.x);
  if (t >= T) return;
  int lo = 0, hi = ndocs;   // the first document that ends behind t
  while (lo < hi) {
    const int mid = lo + ((hi - lo) >> 1);
    if (offsets[mid + 1] > t) hi = mid;
    else lo = mid + 1;
  }
  int4 r = make_int4(0, 0, 0, 0);
  if (lo < ndocs) {
    const int b = max(offsets[lo], 0), e = min(offsets[lo + 1], T);
    if (b <= t && t < e) {
      const int shared = b + (prefix ? min(max(prefix[lo], 0), e - b) : 0);   // keys before it are seen by the whole document
      r = make_int4(b, max(t + 1, shared), t < shared ? b : t, e);
    }
  }
  ranges[t] = r;
}

// ------------------------------------------------------------------------------------------ rotary positions
// Memory bound: q and k are read and written once.  A workgroup takes a few tokens and all their heads, so that a token's angles are
// formed once (in double, as turns, of which the whole ones are dropped before the rounding to float: positions of 2^31 keep an angle good
// to 2^-21) and reach the heads through LDS.  Its first vectors are in flight while it forms them.
constexpr int ROPE_TOKENS = 8;                       // most tokens of a workgroup
constexpr int ROPE_PAIRS = ROPE_AXES_MAX_D / 2;
struct RopeSpectrum { double turns[ROPE_PAIRS]; uint8_t axis[ROPE_PAIRS]; };   // of a pair: turns per position, and which positions
template <typename T> struct RopeSide { const T* in; T* out; int64_t ld_in, ld_out; int cols; };   // the heads of q, or of k

template <typename T>
__global__ __launch_bounds__(256) void rope_axes_kernel(int ntok, int per_block, int half, RopeSide<T> q, RopeSide<T> k, const int32_t* __restrict__ pos,
                                                        RopeSpectrum sp, float sign) {
  constexpr int V = Vec<T>::N, AHEAD = 4;            // vectors in flight per thread
  typedef typename Vec<T>::type vec;
  __shared__ float2 cs[ROPE_TOKENS * ROPE_PAIRS];
  const int t0 = (int)blockIdx.x * per_block, nt = min(per_block, ntok - t0);
  const int qv = q.cols / V, row = qv + k.cols / V;  // vectors of a token
  const int n = nt * row;
  vec x[AHEAD];
  auto place = [&](int i, int& token, int& col, bool& in_q) {
    token = i / row;
    const int v = i - token * row;
    in_q = v < qv;
    col = (in_q ? v : v - qv) * V;
  };
  auto load = [&](int i0) {
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int i = i0 + a * 256;
      if (i < n) {
        int token, col;
        bool in_q;
        place(i, token, col, in_q);
        const RopeSide<T>& s = in_q ? q : k;
        x[a] = *reinterpret_cast<const vec*>(s.in + (t0 + token) * s.ld_in + col);
      }
    }
  };
  load(threadIdx.x);
  for (int i = threadIdx.x; i < nt * half; i += 256) {
    const int token = i / half, p = i - token * half;
    const double turn = sp.turns[p] * (double)pos[(int64_t)sp.axis[p] * ntok + t0 + token];
    float sn, c;
    sincospif((float)(2.0 * (turn - rint(turn))), &sn, &c);
    cs[i] = make_float2(c, sign * sn);
  }
  __syncthreads();
  for (int i0 = threadIdx.x; i0 < n; i0 += AHEAD * 256) {
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int i = i0 + a * 256;
      if (i < n) {
        int token, col;
        bool in_q;
        place(i, token, col, in_q);
        const RopeSide<T>& s = in_q ? q : k;
        const float2* at = cs + token * half + (col / 2) % half;   // a vector lies inside one head
        vec y;
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const float u = to_f(x[a][e]), w = to_f(x[a][e + 1]);
          const float2 r = at[e / 2];
          y[e] = from_f<T>(u * r.x - w * r.y);
          y[e + 1] = from_f<T>(u * r.y + w * r.x);
        }
        *reinterpret_cast<vec*>(s.out + (t0 + token) * s.ld_out + col) = y;
      }
    }
    load(i0 + AHEAD * 256);
  }
}

template <typename T>
hipError_t launch_rope_axes(hipStream_t st, int ntok, int d, const RopeHeads& q, const RopeHeads& k, const int32_t* pos, const RopeSpectrum& sp, int sign) {
  const int per_block = (int)cdiv(ntok, 1024) < ROPE_TOKENS ? (int)cdiv(ntok, 1024) : ROPE_TOKENS;
  const RopeSide<T> a = {(const T*)q.in, (T*)q.out, q.ld_in, q.ld_out, q.n * d}, b = {(const T*)k.in, (T*)k.out, k.ld_in, k.ld_out, k.n * d};
  hipLaunchKernelGGL(rope_axes_kernel<T>, dim3((unsigned)cdiv(ntok, per_block)), dim3(256), 0, st, ntok, per_block, d / 2, a, b, pos, sp, (float)sign);
  return hipGetLastError();
}

}  // namespace

hipError_t doc_ranges(hipStream_t st, int T, int ndocs, const int32_t* offsets, const int32_t* prefix, int32_t* ranges) {
  hipLaunchKernelGGL(doc_ranges_kernel, dim3((unsigned)cdiv(T, 256)), dim3(256), 0, st, T, ndocs, offsets, prefix, (int4*)ranges);
  return hipGetLastError();
}

hipError_t rope_axes(hipStream_t st, DType dt, int T, int d, const RopeHeads& q, const RopeHeads& k, const int32_t* positions, int naxes,
                     const int32_t* sections, int own_spectrum, double base, int sign) {
  RopeSpectrum sp = {};
  int pair = 0;
  for (int a = 0; a < naxes; ++a)
    for (int j = 0; j < sections[a]; ++j, ++pair) {
      const double exponent = own_spectrum ? (double)j / sections[a] : 2.0 * pair / d;
      sp.turns[pair] = pow(base, -exponent) * 0.15915494309189533577;   // 1 / (2 pi)
      sp.axis[pair] = (uint8_t)a;
    }
  return dt == F32    ? launch_rope_axes<float>(st, T, d, q, k, positions, sp, sign)
         : dt == BF16 ? launch_rope_axes<bf16>(st, T, d, q, k, positions, sp, sign)
                      : launch_rope_axes<f16>(st, T, d, q, k, positions, sp, sign);
}

}  // namespace zs
