// Norms of every agent's gradients over all of its tensors, and gradients scaled down to a limit (operators.h).
//
//   norm = sqrt(sum g^2);  f = 1 where norm + eps <= limit, else limit / (norm + eps);  out = f g
//
// Three launches: squares of pieces of kClipPiece elements, a workgroup each; an agent's pieces; the products.  Squares are exact in
// fp64 and summed there.
#include <hip/hip_runtime.h>
#include "operators.h"

namespace pop {
namespace {
namespace clip {

constexpr int kThreads = 256, kTensors = 32;

struct Tensor {
  const void* in;
  void* out;
  int64_t in_matrix, in_row, out_matrix, out_row, elements;
  int cols, dtype;                   // cols 0: an agent's part lies in one piece
  int first;                         // piece of the launch
};
struct Tensors {
  int n, pieces;
  Tensor t[kTensors];
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

struct Place { int agent, tensor; int64_t from; };
__device__ inline Place place_of(const Tensors& a) {
  Place p;
  p.agent = blockIdx.x / a.pieces;
  const int piece = blockIdx.x - p.agent * a.pieces;
  p.tensor = 0;
  while (p.tensor + 1 < a.n && a.t[p.tensor + 1].first <= piece) ++p.tensor;
  p.from = (int64_t)(piece - a.t[p.tensor].first) * kClipPiece;
  return p;
}
__device__ inline int64_t offset(int64_t e, int cols, int64_t row) {
  if (cols == 0) return e;
  const int64_t r = e / cols;
  return r * row + (e - r * cols);
}

template <typename E> __device__ inline double squares(const Tensor& t, const Place& p) {
  const E* in = (const E*)t.in + p.agent * t.in_matrix;
  double s = 0.0;
  for (int i = threadIdx.x; i < kClipPiece; i += kThreads) {
    if (p.from + i >= t.elements) break;
    const double v = (double)(float)in[offset(p.from + i, t.cols, t.in_row)];
    s = fma(v, v, s);
  }
  return s;
}
__global__ void __launch_bounds__(kThreads) k_squares(Tensors a, double* sums, int pieces_of_all, int first) {
  __shared__ double part[4];
  const Place p = place_of(a);
  const Tensor& t = a.t[p.tensor];
  const double s = t.dtype == POP_F32 ? squares<float>(t, p) : t.dtype == POP_BF16 ? squares<__bf16>(t, p) : squares<_Float16>(t, p);
  const double all = sum_of_group(s, part);
  if (threadIdx.x == 0) sums[(int64_t)p.agent * pieces_of_all + first + blockIdx.x % a.pieces] = all;
}

__global__ void __launch_bounds__(kThreads) k_norms(const double* sums, int pieces, double eps, const float* max_norm, float* norms, float* factor) {
  __shared__ double part[4];
  double s = 0.0;
  for (int i = threadIdx.x; i < pieces; i += kThreads) s += sums[(int64_t)blockIdx.x * pieces + i];
  s = sum_of_group(s, part);
  if (threadIdx.x != 0) return;
  const double norm = sqrt(s), above = norm + eps;
  if (norms) norms[blockIdx.x] = (float)norm;
  if (!max_norm) return;
  const float m = max_norm[blockIdx.x];
  const double limit = m < 0.0f ? 0.0 : (double)m;
  factor[blockIdx.x] = above <= limit ? 1.0f : (float)(limit / above);
}

template <typename E> __device__ inline void scale(const Tensor& t, const Place& p, float f) {
  const E* in = (const E*)t.in + p.agent * t.in_matrix;
  E* out = (E*)t.out + p.agent * t.out_matrix;
  for (int i = threadIdx.x; i < kClipPiece; i += kThreads) {
    if (p.from + i >= t.elements) break;
    out[offset(p.from + i, t.cols, t.out_row)] = (E)((float)in[offset(p.from + i, t.cols, t.in_row)] * f);
  }
}
__global__ void __launch_bounds__(kThreads) k_scale(Tensors a, const float* factor) {
  const Place p = place_of(a);
  const Tensor& t = a.t[p.tensor];
  const float f = factor[p.agent];
  if (t.dtype == POP_F32) scale<float>(t, p, f);
  else if (t.dtype == POP_BF16) scale<__bf16>(t, p, f);
  else scale<_Float16>(t, p, f);
}

int64_t all_pieces(int n, const pop_gradient* g) {
  int64_t sum = 0;
  for (int k = 0; k < n; ++k) sum += clip_pieces((int64_t)g[k].rows * g[k].cols);
  return sum;
}

Tensors tensors_of(const ClipCall& c, int from, int to) {
  Tensors a = {};
  for (int k = from; k < to; ++k) {
    const pop_gradient& g = c.grads[k];
    Tensor& t = a.t[a.n++];
    t.in = g.grad.data; t.in_matrix = g.grad.matrix; t.in_row = g.grad.row;
    t.out = g.out.data; t.out_matrix = g.out.matrix; t.out_row = g.out.row;
    t.elements = (int64_t)g.rows * g.cols;
    t.cols = g.rows == 1 || (g.grad.row == g.cols && (!c.max_norm || g.out.row == g.cols)) ? 0 : g.cols;
    t.dtype = g.dtype;
    t.first = a.pieces;
    a.pieces += (int)clip_pieces(t.elements);
  }
  return a;
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
  int first = 0;
  for (int k = 0; k < c.n; k += kTensors) {
    const Tensors a = tensors_of(c, k, k + kTensors < c.n ? k + kTensors : c.n);
    k_squares<<<(unsigned)(a.pieces * c.P), kThreads, 0, s>>>(a, sums, pieces, first);
    first += a.pieces;
  }
  k_norms<<<(unsigned)c.P, kThreads, 0, s>>>(sums, pieces, c.eps, c.max_norm, c.norms, factor);
  if (c.max_norm)
    for (int k = 0; k < c.n; k += kTensors) {
      const Tensors a = tensors_of(c, k, k + kTensors < c.n ? k + kTensors : c.n);
      k_scale<<<(unsigned)(a.pieces * c.P), kThreads, 0, s>>>(a, factor);
    }
  return hipGetLastError();
}

}  // namespace pop
