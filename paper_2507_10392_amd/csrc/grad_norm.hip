// The norm of many gradient tensors taken together, the factor that clips them, and the tensors times that factor.
//
// Memory bound: every element is read once for the norm, and once more and written for the clipping, which cannot begin before.  A launch takes up to
// 160 tensors, whatever their types and sizes, in its arguments (no table on the device that could be out of date); its workgroups take pieces of them
// of one size, which grows with the total so that there are some thousand pieces at most.  A tensor's pieces begin at multiples of 16 bytes behind its
// first aligned element, whose predecessors belong to the first piece.
//
// Squares are formed and added in 64 bits: gradients may be larger than 2^64 or smaller than 2^-75, whose squares fp32 does not hold, and a sum over
// 10^9 elements keeps its digits.  That costs two instructions per element, of which the memory leaves time for ten.  The pieces' sums are added in
// their order by a workgroup of a second kernel, so a repeat gives the same bits.  405 M fp32 in 18 tensors: norm 290 to 300 us, clipping 560 to 606, both at
// 5.3 to 5.8 TB/s; 26 tensors of 1.6 M together 4 + 2 us.  Clipping in the opposite order, for what the norm left in the last-level cache, was no faster.
#include "kernels.h"

#include <algorithm>
#include <cmath>

namespace zs {
namespace {

constexpr int PACK = 160;          // tensors of a launch: its arguments stay below 4096 bytes (with sizes and first pieces apart 128 would; 300 tensors: 116 us, 125)
constexpr int THREADS = 256;
constexpr int AHEAD = 8;           // vectors that a thread has in flight
struct TensorPack {
  const void* in[PACK];
  void* out[PACK];
  uint64_t place[PACK];            // elements, below 2^51, and behind them the tensor's first of the launch's pieces, below 2^13
  uint8_t type[PACK];
  int32_t count, pieces;
  int64_t piece;                   // bytes
};
static_assert(sizeof(TensorPack) + sizeof(void*) <= 4096, "");
constexpr int MOST_PIECES = 4096;  // and one more of every tensor
static_assert(MOST_PIECES + PACK < 1 << 13, "");
__device__ __forceinline__ int first_of(const TensorPack& p, int t) { return (int)(p.place[t] & 8191); }
__device__ __forceinline__ int64_t size_of(const TensorPack& p, int t) { return (int64_t)(p.place[t] >> 13); }

// The tensor that a piece belongs to: the last one whose first piece is not behind it.
__device__ __forceinline__ int tensor_of(const TensorPack& p, int piece) {
  const int lane = threadIdx.x & 63;
  int at = -1;
#pragma unroll
  for (int i = 0; i < (PACK + 63) / 64; ++i) {
    const int t = lane + 64 * i;
    at += __popcll(__ballot(t < p.count && first_of(p, min(t, PACK - 1)) <= piece));
  }
  return __builtin_amdgcn_readfirstlane(at);
}

// The elements begin .. end-1 of a tensor, of which body .. body + 16-byte vectors are aligned.
struct Piece { int64_t begin, body, end; };
template <typename E> __device__ __forceinline__ Piece piece_of(const E* x, int64_t n, int64_t piece, int k) {
  const int64_t head = (int64_t)((16 - ((uintptr_t)x & 15)) & 15) / (int64_t)sizeof(E), step = piece / (int64_t)sizeof(E);
  const int64_t body = head + k * step, end = body + step;
  return Piece{k == 0 ? 0 : min(body, n), min(body, n), min(end, n)};
}

template <typename E> __device__ __forceinline__ double sum_squares(const E* __restrict__ x, const Piece& p) {
  typedef typename Vec<E>::type vec;
  constexpr int N = Vec<E>::N;
  double s[2] = {0.0, 0.0};
  auto add = [&](int i, float v) { s[i & 1] = fma((double)v, (double)v, s[i & 1]); };
  const vec* v = reinterpret_cast<const vec*>(x + p.body);
  const int64_t vectors = (p.end - p.body) / N;
  int64_t i = threadIdx.x;
  for (; i + (AHEAD - 1) * THREADS < vectors; i += AHEAD * THREADS) {
    vec a[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) a[j] = v[i + j * THREADS];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) add(e, (float)a[j][e]);
  }
  for (; i < vectors; i += THREADS) {
    const vec a = v[i];
#pragma unroll
    for (int e = 0; e < N; ++e) add(e, (float)a[e]);
  }
  const int64_t tail = p.body + vectors * N;
  if (p.begin + threadIdx.x < p.body) add(0, to_f(x[p.begin + threadIdx.x]));
  if (tail + threadIdx.x < p.end) add(1, to_f(x[tail + threadIdx.x]));
  return s[0] + s[1];
}

template <int NW> __device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int i = 0; i < NW; ++i) t += red[i];
  return t;
}

__global__ __launch_bounds__(THREADS) void grad_norm_kernel(TensorPack p, double* __restrict__ sums) {
  __shared__ double red[THREADS / 64];
  const int t = tensor_of(p, blockIdx.x), k = (int)blockIdx.x - first_of(p, t), type = p.type[t];
  const void* x = p.in[t];
  const int64_t n = size_of(p, t);
  double s;
  if (type == F32) s = sum_squares((const float*)x, piece_of((const float*)x, n, p.piece, k));
  else if (type == BF16) s = sum_squares((const bf16*)x, piece_of((const bf16*)x, n, p.piece, k));
  else s = sum_squares((const f16*)x, piece_of((const f16*)x, n, p.piece, k));
  s = block_sum<THREADS / 64>(s, red);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// The sums' sum, the norm, the factor and whether the norm is finite.
__global__ __launch_bounds__(THREADS) void grad_factor_kernel(int64_t n, const double* __restrict__ sums, double scale, double max_norm, double* sumsq, float* norm,
                                                              float* factor, int* overflow) {
  __shared__ double red[THREADS / 64];
  double s = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < n; i += THREADS) s += sums[i];
  s = block_sum<THREADS / 64>(s, red);
  if (threadIdx.x) return;
  const double len = scale * sqrt(s);
  const bool fine = len <= 1.7976931348623157e308;   // neither inf nor NaN
  if (sumsq) *sumsq = s;
  if (norm) *norm = (float)len;
  if (factor) *factor = fine && len > max_norm ? (float)(max_norm / len) : 1.f;
  if (overflow && !fine) atomicOr(overflow, 1);
}

template <typename E> __device__ __forceinline__ void scale_piece(const E* x, E* y, const Piece& p, float f) {
  typedef typename Vec<E>::type vec;
  constexpr int N = Vec<E>::N;
  if (((uintptr_t)x ^ (uintptr_t)y) & 15) {   // no place where both are aligned
    for (int64_t i = p.begin + threadIdx.x; i < p.end; i += THREADS) y[i] = from_f<E>(fp32_value(to_f(x[i]) * f));
    return;
  }
  const vec* v = reinterpret_cast<const vec*>(x + p.body);
  vec* w = reinterpret_cast<vec*>(y + p.body);
  const int64_t vectors = (p.end - p.body) / N;
  auto times = [&](vec a) {
#pragma unroll
    for (int e = 0; e < N; ++e) a[e] = from_f<E>(fp32_value((float)a[e] * f));
    return a;
  };
  int64_t i = threadIdx.x;
  for (; i + (AHEAD - 1) * THREADS < vectors; i += AHEAD * THREADS) {
    vec a[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) a[j] = v[i + j * THREADS];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) w[i + j * THREADS] = times(a[j]);
  }
  for (; i < vectors; i += THREADS) w[i] = times(v[i]);
  const int64_t tail = p.body + vectors * N;
  if (p.begin + threadIdx.x < p.body) y[p.begin + threadIdx.x] = from_f<E>(fp32_value(to_f(x[p.begin + threadIdx.x]) * f));
  if (tail + threadIdx.x < p.end) y[tail + threadIdx.x] = from_f<E>(fp32_value(to_f(x[tail + threadIdx.x]) * f));
}

__global__ __launch_bounds__(THREADS) void grad_scale_kernel(TensorPack p, const float* __restrict__ factor) {
  const float f = *factor;
  const int t = tensor_of(p, blockIdx.x), k = (int)blockIdx.x - first_of(p, t), type = p.type[t];
  const void* x = p.in[t];
  void* y = p.out[t];
  if (f == 1.f && x == y) return;
  const int64_t n = size_of(p, t);
  if (type == F32) scale_piece((const float*)x, (float*)y, piece_of((const float*)x, n, p.piece, k), f);
  else if (type == BF16) scale_piece((const bf16*)x, (bf16*)y, piece_of((const bf16*)x, n, p.piece, k), f);
  else scale_piece((const f16*)x, (f16*)y, piece_of((const f16*)x, n, p.piece, k), f);
}

int64_t bytes_of(const GradTensor& t) { return t.n * (t.dtype == F32 ? 4 : 2); }
// Pieces of 16 KB, larger ones where that would be more than MOST_PIECES of them.
int64_t piece_bytes(const GradTensor* t, int count) {
  int64_t total = 0, piece = 16 << 10;
  for (int i = 0; i < count; ++i) total += bytes_of(t[i]);
  while (total / piece > MOST_PIECES) piece *= 2;
  return piece;
}
int64_t pieces_of(const GradTensor& t, int64_t piece) {   // up to 15 bytes may lie before the first
  const int64_t size = t.dtype == F32 ? 4 : 2, head = std::min<int64_t>(t.n, (int64_t)((16 - ((uintptr_t)t.in & 15)) & 15) / size);
  return t.n == 0 ? 0 : std::max<int64_t>(1, cdiv((t.n - head) * size, piece));
}

// f(pack, pieces before it) for groups of tensors.
template <typename F> hipError_t for_packs(const GradTensor* t, int count, F&& f) {
  TensorPack p = {};
  p.piece = piece_bytes(t, count);
  int64_t before = 0;
  for (int i = 0; i < count; ++i) {
    const int64_t k = pieces_of(t[i], p.piece);
    if (k) {
      const int c = p.count++;
      p.in[c] = t[i].in; p.out[c] = t[i].out; p.type[c] = (uint8_t)t[i].dtype;
      p.place[c] = (uint64_t)t[i].n << 13 | (uint64_t)p.pieces;
      p.pieces += (int32_t)k;
    }
    if (p.count == PACK || (i + 1 == count && p.count)) {
      const hipError_t e = f(p, before);
      if (e != hipSuccess) return e;
      before += p.pieces;
      p.count = p.pieces = 0;
    }
  }
  return hipSuccess;
}
}  // namespace

int64_t grad_norm_pieces(const GradTensor* t, int count) {
  const int64_t piece = piece_bytes(t, count);
  int64_t n = 0;
  for (int i = 0; i < count; ++i) n += pieces_of(t[i], piece);
  return n;
}
hipError_t grad_norm(hipStream_t st, const GradTensor* t, int count, const GradClip& c, double* sums) {
  const hipError_t e = for_packs(t, count, [&](const TensorPack& p, int64_t before) {
    hipLaunchKernelGGL(grad_norm_kernel, dim3((unsigned)p.pieces), dim3(THREADS), 0, st, p, sums + before);
    return hipGetLastError();
  });
  return e != hipSuccess ? e : grad_factor(st, grad_norm_pieces(t, count), sums, c);
}
hipError_t grad_factor(hipStream_t st, int64_t n, const double* sums, const GradClip& c) {
  hipLaunchKernelGGL(grad_factor_kernel, dim3(1), dim3(THREADS), 0, st, n, sums, (double)c.scale, (double)c.max_norm, c.sumsq, c.norm, c.factor, c.overflow);
  return hipGetLastError();
}
hipError_t grad_scale(hipStream_t st, const GradTensor* t, int count, const float* factor) {
  return for_packs(t, count, [&](const TensorPack& p, int64_t) {
    hipLaunchKernelGGL(grad_scale_kernel, dim3((unsigned)p.pieces), dim3(THREADS), 0, st, p, factor);
    return hipGetLastError();
  });
}

}  // namespace zs
