// Norms of every agent's gradients over all of its tensors, and gradients scaled down to a limit (operators.h).
//
//   norm = sqrt(sum g^2);  f = 1 where norm + eps <= limit, else limit / (norm + eps);  out = f g
//
// Squares of pieces of kClipPiece elements, a workgroup each, exact in fp64 and summed there; then the products, whose workgroups sum an
// agent's pieces for themselves where it has up to kFew, so that two launches do (10 agents of six tensors: 39 -> 28 us a call, most of it the
// host's), and a launch for the norms in between where it has more.  Bound by memory: gradients are read twice and written once, with
// the second reading from the end, where it finds in the last cache what was read last: 4 agents of 30 million fp32 elements in 18 tensors,
// 246 us, 1.45 GB at 5.9 TB/s.  Results past the caches (kPast): 246 against 277 us there.
#include <hip/hip_runtime.h>
#include "operators.h"

namespace pop {
namespace {
namespace clip {

constexpr int kThreads = 256;
constexpr int kFew = kThreads;         // sums of pieces that a workgroup reads at once

// Pieces from which on results are stored past the caches, which hold what is about to be read again: a quarter of the 256 MB of the last one.
constexpr int kPast = (64 << 20) / (4 * kClipPiece);

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

struct Tensor {
  const void* in;
  void* out;
  int64_t in_matrix, in_row, out_matrix, out_row, elements;
  int cols, dtype;                   // cols 0: an agent's part lies in one piece
  int first;                         // piece of the launch
  int wide;                          // vectors of 16 bytes end where rows end
};
template <int N> struct Tensors {
  int n, pieces;
  Tensor t[N];
};

__device__ inline double sum_of_wave(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
// The sum over a workgroup, in every lane.
__device__ inline double sum_of_group(double v, double* part) {
  v = sum_of_wave(v);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}

struct Place { int agent, tensor, count; int64_t from; };
template <int N> __device__ inline Place place_of(const Tensors<N>& a, int block) {
  Place p;
  p.agent = block / a.pieces;
  const int piece = block - p.agent * a.pieces;
  p.tensor = 0;
  while (p.tensor + 1 < a.n && a.t[p.tensor + 1].first <= piece) ++p.tensor;
  p.from = (int64_t)(piece - a.t[p.tensor].first) * kClipPiece;
  const int64_t left = a.t[p.tensor].elements - p.from;
  p.count = left < kClipPiece ? (int)left : kClipPiece;
  return p;
}

// Where the elements of a piece lie: element i at `at`(i) from the agent's part.
struct Rows {
  int64_t row, first;
  unsigned cols, skip;
  __device__ inline Rows(int64_t from, int cols, int64_t row) : row(row), first(from), cols(cols), skip(0) {
    if (cols != 0) {
      first = from / cols;
      skip = (unsigned)(from - first * cols);
    }
  }
  __device__ inline int64_t at(int i) const {
    if (cols == 0) return first + i;
    const unsigned r = (skip + i) / cols;                            // skip < 2^31, i < 2^13
    return (first + r) * row + (skip + i - r * cols);
  }
};

// What a thread has of a piece: vectors of 16 bytes threadIdx.x, threadIdx.x + kThreads, ..; where rows do not allow them, and behind the
// last whole one, the vector's elements one by one.  Vectors need no more alignment than elements.
template <typename E> struct Part {
  static constexpr int kVec = 16 / sizeof(E), kEach = kClipPiece / kVec / kThreads;
  u32x4 v[kEach];
  static __device__ inline int at(int k) { return (int)(threadIdx.x + k * kThreads) * kVec; }
  __device__ inline void load(const E* in, const Rows& rows, int count, bool wide) {
    if (wide && count == kClipPiece) {
#pragma unroll
      for (int k = 0; k < kEach; ++k) __builtin_memcpy(&v[k], in + rows.at(at(k)), 16);
    } else {
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        v[k] = u32x4{0, 0, 0, 0};
        if (wide && at(k) + kVec <= count) {
          __builtin_memcpy(&v[k], in + rows.at(at(k)), 16);
        } else {
          E e[kVec];
#pragma unroll
          for (int i = 0; i < kVec; ++i) e[i] = at(k) + i < count ? in[rows.at(at(k) + i)] : (E)0.0f;
          __builtin_memcpy(&v[k], e, 16);
        }
      }
    }
  }
  template <bool PAST> __device__ inline void store(E* out, const Rows& rows, int count, bool wide) const {
    typedef u32x4 Anywhere __attribute__((aligned(2)));
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (wide && at(k) + kVec <= count) {
        Anywhere* to = (Anywhere*)(out + rows.at(at(k)));
        if constexpr (PAST) __builtin_nontemporal_store(v[k], to);
        else *to = v[k];
      } else {
        E e[kVec];
        __builtin_memcpy(e, &v[k], 16);
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          if (at(k) + i < count) out[rows.at(at(k) + i)] = e[i];
      }
    }
  }
};

template <typename E> __device__ inline double squares(const Tensor& t, const Place& p) {
  Part<E> part;
  part.load((const E*)t.in + p.agent * t.in_matrix, Rows(p.from, t.cols, t.in_row), p.count, t.wide);
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < Part<E>::kEach; ++k) {
    E e[Part<E>::kVec];
    __builtin_memcpy(e, &part.v[k], 16);
#pragma unroll
    for (int i = 0; i < Part<E>::kVec; ++i) {
      const double v = (double)(float)e[i];
      s = fma(v, v, s);
    }
  }
  return s;
}
template <int N> __global__ void __launch_bounds__(kThreads) k_squares(Tensors<N> a, double* sums, int pieces_of_all, int first) {
  __shared__ double part[4];
  const Place p = place_of(a, blockIdx.x);
  const Tensor& t = a.t[p.tensor];
  const double s = t.dtype == POP_F32 ? squares<float>(t, p) : t.dtype == POP_BF16 ? squares<__bf16>(t, p) : squares<_Float16>(t, p);
  const double all = sum_of_group(s, part);
  if (threadIdx.x == 0) sums[(int64_t)p.agent * pieces_of_all + first + (int)blockIdx.x - p.agent * a.pieces] = all;
}

// The sums of an agent's pieces, and what becomes of them.
struct Limits {
  const double* sums;
  int pieces;
  double eps;
  const float* max_norm;
  float* norms;
};
__device__ inline double norm_of(const Limits& l, int agent, double* part) {
  double s = 0.0;
  for (int i = threadIdx.x; i < l.pieces; i += kThreads) s += l.sums[(int64_t)agent * l.pieces + i];
  return sqrt(sum_of_group(s, part));
}
__device__ inline float factor_of(const Limits& l, int agent, double norm) {
  const float m = l.max_norm[agent];
  const double limit = m < 0.0f ? 0.0 : (double)m, above = norm + l.eps;
  return above <= limit ? 1.0f : (float)(limit / above);
}
__global__ void __launch_bounds__(kThreads) k_norms(Limits l, float* factor) {
  __shared__ double part[4];
  const double norm = norm_of(l, blockIdx.x, part);
  if (threadIdx.x != 0) return;
  if (l.norms) l.norms[blockIdx.x] = (float)norm;
  if (factor) factor[blockIdx.x] = factor_of(l, blockIdx.x, norm);
}

template <typename E, bool PAST> __device__ inline void scale(const Tensor& t, const Place& p, float f) {
  const E* in = (const E*)t.in + p.agent * t.in_matrix;
  E* out = (E*)t.out + p.agent * t.out_matrix;
  if (f == 1.0f && in == out) return;                                // (the boundary has checked that strides are the same then)
  Part<E> part;
  part.load(in, Rows(p.from, t.cols, t.in_row), p.count, t.wide);
#pragma unroll
  for (int k = 0; k < Part<E>::kEach; ++k) {
    E e[Part<E>::kVec];
    __builtin_memcpy(e, &part.v[k], 16);
#pragma unroll
    for (int i = 0; i < Part<E>::kVec; ++i) e[i] = (E)((float)e[i] * f);
    __builtin_memcpy(&part.v[k], e, 16);
  }
  part.template store<PAST>(out, Rows(p.from, t.cols, t.out_row), p.count, t.wide);
}
// factor NULL: every workgroup finds its agent's norm for itself, and the one with the agent's first piece of all writes it.
template <int N, bool PAST> __global__ void __launch_bounds__(kThreads) k_scale(Tensors<N> a, Limits l, const float* factor, int first) {
  __shared__ double part[4];
  const int block = gridDim.x - 1 - blockIdx.x;                      // what was read last may still be in a cache
  const Place p = place_of(a, block);
  const Tensor& t = a.t[p.tensor];
  float f;
  if (factor) {
    f = factor[p.agent];
  } else {
    const double norm = norm_of(l, p.agent, part);
    f = factor_of(l, p.agent, norm);
    if (l.norms && threadIdx.x == 0 && first == 0 && block == p.agent * a.pieces) l.norms[p.agent] = (float)norm;
  }
  if (t.dtype == POP_F32) scale<float, PAST>(t, p, f);
  else if (t.dtype == POP_BF16) scale<__bf16, PAST>(t, p, f);
  else scale<_Float16, PAST>(t, p, f);
}

int64_t all_pieces(int n, const pop_gradient* g) {
  int64_t sum = 0;
  for (int k = 0; k < n; ++k) sum += clip_pieces((int64_t)g[k].rows * g[k].cols);
  return sum;
}

template <int N> Tensors<N> tensors_of(const ClipCall& c, int from) {
  Tensors<N> a;
  a.n = a.pieces = 0;
  for (int k = from; k < c.n && k < from + N; ++k) {
    const pop_gradient& g = c.grads[k];
    Tensor& t = a.t[a.n++];
    t.in = g.grad.data; t.in_matrix = g.grad.matrix; t.in_row = g.grad.row;
    t.out = g.out.data; t.out_matrix = g.out.matrix; t.out_row = g.out.row;
    t.elements = (int64_t)g.rows * g.cols;
    t.cols = g.rows == 1 || (g.grad.row == g.cols && (!c.max_norm || g.out.row == g.cols)) ? 0 : g.cols;
    t.dtype = g.dtype;
    t.wide = t.cols % (g.dtype == POP_F32 ? 4 : 8) == 0;
    t.first = a.pieces;
    a.pieces += (int)clip_pieces(t.elements);
  }
  return a;
}

template <int N> void launch(const ClipCall& c, const Limits& l, float* factor, hipStream_t s) {
  const bool few = c.max_norm && l.pieces <= kFew, past = (int64_t)l.pieces * c.P >= kPast;
  int first = 0;
  Tensors<N> a;
  for (int k = 0; k < c.n; k += N) {
    a = tensors_of<N>(c, k);
    k_squares<N><<<(unsigned)(a.pieces * c.P), kThreads, 0, s>>>(a, (double*)l.sums, l.pieces, first);
    first += a.pieces;
  }
  if (!few) k_norms<<<(unsigned)c.P, kThreads, 0, s>>>(l, c.max_norm ? factor : nullptr);
  if (!c.max_norm) return;
  first = 0;
  for (int k = 0; k < c.n; k += N) {
    if (c.n > N) a = tensors_of<N>(c, k);
    if (past) k_scale<N, true><<<(unsigned)(a.pieces * c.P), kThreads, 0, s>>>(a, l, few ? nullptr : factor, first);
    else k_scale<N, false><<<(unsigned)(a.pieces * c.P), kThreads, 0, s>>>(a, l, few ? nullptr : factor, first);
    first += a.pieces;
  }
}

}  // namespace clip
}  // namespace

int64_t clip_workspace_bytes(int64_t P, int n, const pop_gradient* grads) {
  return (P * (clip::all_pieces(n, grads) * 8 + 4) + 255) / 256 * 256;
}

hipError_t launch_clip(const ClipCall& c, void* ws, hipStream_t s) {
  using namespace clip;
  const int pieces = (int)all_pieces(c.n, c.grads);
  double* sums = (double*)ws;
  float* factor = (float*)(sums + (int64_t)c.P * pieces);
  const Limits l = {sums, pieces, c.eps, c.max_norm, c.norms};
  if (c.n <= 8) clip::launch<8>(c, l, factor, s);
  else clip::launch<32>(c, l, factor, s);
  return hipGetLastError();
}

}  // namespace pop
