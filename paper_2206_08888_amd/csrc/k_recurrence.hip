// Gated linear recurrence over sequences, its backward pass, and single steps (operators.h).
//
//   a_t = sigmoid(g_t + bias),  h_t = a_t keep_t h_{t-1} + (1 - a_t) x_t;  keep_t = 0 at resets
//   backward, d_t = dL/dh_t:  d_t = dy_t + a_{t+1} keep_{t+1} d_{t+1};  dx_t = d_t (1 - a_t);
//   dg_t = d_t (keep_t h_{t-1} - x_t) a_t (1 - a_t);  dbias = sum dg;  dh0 = a_0 keep_0 d_0
//
// Both directions are scans: a run of steps maps the state s in front of it to A s + H, and such maps compose.  A run
// with a reset has A = -0: then s is left out, not multiplied (it may be NaN or infinite).  A
// sequence is cut into chunks of kRecurChunk steps; one launch finds A and H of every chunk, one carries the state
// over the chunks, one computes the outputs of every chunk from the state in front of it.
#include <hip/hip_runtime.h>
#include "operators.h"

namespace pop {
namespace {
namespace recur {

template <typename E> __device__ inline float load(const pop_sequence& s, int64_t at) { return (float)((const E*)s.data)[at]; }
template <typename E> __device__ inline void store(const pop_sequence& s, int64_t at, float v) { ((E*)s.data)[at] = (E)v; }

// sigmoid(z) and 1 - sigmoid(z), each to fp32's precision
struct Gate { float a, b; };
__device__ inline Gate gate(float z) {
  const float e = __expf(-fabsf(z)), big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  return z >= 0.0f ? Gate{big, small} : (z < 0.0f ? Gate{small, big} : Gate{z, z});   // NaN stays NaN
}

__device__ inline bool cut(float A) { return __float_as_uint(A) >> 31; }                    // the run has a reset
__device__ inline float apply(float A, float H, float s) { return cut(A) ? H : fmaf(A, s, H); }

// one lane's channel of one sequence
struct Lane {
  int p, b, c;
  int64_t row;                                        // p * B + b
  int len;
  float bias;
};
__device__ inline bool lane_of(const RecurArgs& a, Lane& l) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (int64_t)a.P * a.B * a.C) return false;
  l.c = (int)(i % a.C);
  l.row = i / a.C;
  l.p = (int)(l.row / a.B);
  l.b = (int)(l.row % a.B);
  l.len = a.lengths ? min(max(a.lengths[l.row], 0), a.T) : a.T;
  l.bias = a.bias ? a.bias[(int64_t)l.p * a.C + l.c] : 0.0f;
  return true;
}
__device__ inline int64_t base(const pop_sequence& s, const Lane& l) { return l.p * s.agent + l.b * s.row + l.c; }
__device__ inline bool is_reset(const RecurArgs& a, const Lane& l, int t) {
  return a.reset.data && ((const uint8_t*)a.reset.data)[l.p * a.reset.agent + l.b * a.reset.row + (int64_t)t * a.reset.step] != 0;
}

constexpr int kLanes = 256;

// workspace: A, H of every chunk [rows, chunks, C] each; backward: the gradient behind every chunk, and the sums of
// dg over each chunk, in the same layout
template <typename E>
__global__ void __launch_bounds__(kLanes) k_forward_chunks(RecurArgs a, int chunks) {
  Lane l;
  if (!lane_of(a, l)) return;
  const int k = blockIdx.y, t0 = k * kRecurChunk, t1 = min(t0 + kRecurChunk, l.len);
  float A = 1.0f, H = 0.0f;
  for (int t = t0; t < t1; ++t) {
    const Gate q = gate(load<E>(a.g, base(a.g, l) + t * a.g.step) + l.bias);
    const float u = q.b * load<E>(a.x, base(a.x, l) + t * a.x.step);
    const bool r = is_reset(a, l, t);
    A = r ? -0.0f : A * q.a;
    H = r ? u : fmaf(q.a, H, u);
  }
  const int64_t n = (int64_t)a.P * a.B * chunks * a.C, at = (l.row * chunks + k) * a.C + l.c;
  a.ws[at] = A;
  a.ws[n + at] = H;
}

__global__ void __launch_bounds__(kLanes) k_forward_carry(RecurArgs a, int chunks, float* states) {
  Lane l;
  if (!lane_of(a, l)) return;
  const int64_t n = (int64_t)a.P * a.B * chunks * a.C;
  float h = a.h0 ? a.h0[l.row * a.C + l.c] : 0.0f;
  for (int k = 0; k < chunks; ++k) {
    const int64_t at = (l.row * chunks + k) * a.C + l.c;
    const float A = a.ws[at], H = a.ws[n + at];
    states[at] = h;
    if (k * kRecurChunk < l.len) h = apply(A, H, h);
  }
  if (a.h_last) a.h_last[l.row * a.C + l.c] = h;
}

template <typename E>
__global__ void __launch_bounds__(kLanes) k_forward(RecurArgs a, int chunks, const float* states) {
  Lane l;
  if (!lane_of(a, l)) return;
  const int k = blockIdx.y, t0 = k * kRecurChunk, end = min(t0 + kRecurChunk, a.T);
  float h = states[(l.row * chunks + k) * a.C + l.c];
  for (int t = t0; t < end; ++t) {
    if (t < l.len) {
      const Gate q = gate(load<E>(a.g, base(a.g, l) + t * a.g.step) + l.bias);
      const float u = q.b * load<E>(a.x, base(a.x, l) + t * a.x.step);
      h = is_reset(a, l, t) ? u : fmaf(q.a, h, u);
    }
    store<E>(a.y, base(a.y, l) + t * a.y.step, t < l.len ? h : 0.0f);
  }
}

__global__ void __launch_bounds__(kLanes) k_no_steps(const float* from, float* to, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) to[i] = from ? from[i] : 0.0f;
}

template <typename E>
__global__ void __launch_bounds__(kLanes) k_backward_chunks(RecurArgs a, int chunks) {
  Lane l;
  if (!lane_of(a, l)) return;
  const int k = blockIdx.y, t0 = k * kRecurChunk, t1 = min(t0 + kRecurChunk, l.len);
  float A = 1.0f, H = 0.0f;                           // what leaves the chunk in front: A d + H
  for (int t = t1 - 1; t >= t0; --t) {
    const Gate q = gate(load<E>(a.g, base(a.g, l) + t * a.g.step) + l.bias);
    const float dy = load<E>(a.dy, base(a.dy, l) + t * a.dy.step);
    const bool r = is_reset(a, l, t);
    A = r ? -0.0f : A * q.a;
    H = r ? 0.0f : q.a * (H + dy);
  }
  const int64_t n = (int64_t)a.P * a.B * chunks * a.C, at = (l.row * chunks + k) * a.C + l.c;
  a.ws[at] = A;
  a.ws[n + at] = H;
}

__global__ void __launch_bounds__(kLanes) k_backward_carry(RecurArgs a, int chunks) {
  Lane l;
  if (!lane_of(a, l)) return;
  const int64_t n = (int64_t)a.P * a.B * chunks * a.C;
  float d = a.dh_last ? a.dh_last[l.row * a.C + l.c] : 0.0f;
  for (int k = chunks - 1; k >= 0; --k) {
    const int64_t at = (l.row * chunks + k) * a.C + l.c;
    const float A = a.ws[at], H = a.ws[n + at];
    a.ws[at] = d;
    if (k * kRecurChunk < l.len) d = apply(A, H, d);
  }
  if (a.dh0) a.dh0[l.row * a.C + l.c] = d;
}

// Outputs of a chunk: its states are found again from the one in front of it, a run of kRun steps at a time.
constexpr int kRun = 16, kRuns = kRecurChunk / kRun;

template <typename E>
__global__ void __launch_bounds__(kLanes) k_backward(RecurArgs a, int chunks) {
  Lane l;
  if (!lane_of(a, l)) return;
  const int k = blockIdx.y, t0 = k * kRecurChunk, end = min(t0 + kRecurChunk, a.T);
  const int64_t n = (int64_t)a.P * a.B * chunks * a.C, at = (l.row * chunks + k) * a.C + l.c;
  const auto step = [&](int t, float h) {
    const Gate q = gate(load<E>(a.g, base(a.g, l) + t * a.g.step) + l.bias);
    const float u = q.b * load<E>(a.x, base(a.x, l) + t * a.x.step);
    return is_reset(a, l, t) ? u : fmaf(q.a, h, u);
  };
  float front[kRuns];
  float h = a.states[at], d = a.ws[at], sum = 0.0f;
#pragma unroll
  for (int r = 0; r < kRuns; ++r) {
    front[r] = h;
    for (int t = t0 + r * kRun; t < min(t0 + (r + 1) * kRun, l.len); ++t) h = step(t, h);
  }
  for (int t = max(t0, l.len); t < end; ++t) {
    store<E>(a.dx, base(a.dx, l) + t * a.dx.step, 0.0f);
    store<E>(a.dg, base(a.dg, l) + t * a.dg.step, 0.0f);
  }
#pragma unroll
  for (int r = kRuns - 1; r >= 0; --r) {
    const int s0 = t0 + r * kRun;
    float before[kRun];
    h = front[r];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      before[i] = h;
      if (s0 + i < l.len) h = step(s0 + i, h);
    }
#pragma unroll
    for (int i = kRun - 1; i >= 0; --i) {
      const int t = s0 + i;
      if (t >= l.len) continue;
      const Gate q = gate(load<E>(a.g, base(a.g, l) + t * a.g.step) + l.bias);
      const float x = load<E>(a.x, base(a.x, l) + t * a.x.step);
      const bool r0 = is_reset(a, l, t);
      d += load<E>(a.dy, base(a.dy, l) + t * a.dy.step);
      const float dg = d * ((r0 ? 0.0f : before[i]) - x) * (q.a * q.b);
      store<E>(a.dx, base(a.dx, l) + t * a.dx.step, d * q.b);
      store<E>(a.dg, base(a.dg, l) + t * a.dg.step, dg);
      sum += dg;
      d = r0 ? 0.0f : d * q.a;
    }
  }
  a.ws[n + at] = sum;
}

__global__ void __launch_bounds__(kLanes) k_bias_sum(const float* sums, float* dbias, int64_t n, int C, int64_t parts) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  const float* s = sums + i / C * parts * C + i % C;
  float v = 0.0f;
  for (int64_t k = 0; k < parts; ++k) v += s[k * C];
  dbias[i] = v;
}

template <typename E>
__global__ void __launch_bounds__(kLanes) k_step(RecurArgs a) {
  Lane l;
  if (!lane_of(a, l)) return;
  const int slot = a.slots ? a.slots[l.row] : l.b;
  float h = 0.0f;
  if (slot >= 0 && slot < a.n_slots) {
    float* state = a.state + ((int64_t)l.p * a.n_slots + slot) * a.C + l.c;
    const Gate q = gate(load<E>(a.g, base(a.g, l)) + l.bias);
    const float u = q.b * load<E>(a.x, base(a.x, l));
    h = is_reset(a, l, 0) ? u : fmaf(q.a, *state, u);
    *state = h;
  }
  store<E>(a.y, base(a.y, l), h);
}

unsigned blocks(int64_t n) { return (unsigned)((n + kLanes - 1) / kLanes); }

template <typename E> hipError_t forward(const RecurArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.P * a.B * a.C;
  const int chunks = (int)recur_chunks(a.T);
  float* states = a.states ? a.states : a.ws + 2 * n * chunks;
  if (chunks == 0) {
    if (a.h_last) k_no_steps<<<blocks(n), kLanes, 0, s>>>(a.h0, a.h_last, n);
    return hipGetLastError();
  }
  k_forward_chunks<E><<<dim3(blocks(n), chunks), kLanes, 0, s>>>(a, chunks);
  k_forward_carry<<<blocks(n), kLanes, 0, s>>>(a, chunks, states);
  k_forward<E><<<dim3(blocks(n), chunks), kLanes, 0, s>>>(a, chunks, states);
  return hipGetLastError();
}

template <typename E> hipError_t backward(const RecurArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.P * a.B * a.C, nb = (int64_t)a.P * a.C;
  const int chunks = (int)recur_chunks(a.T);
  if (chunks == 0) {
    if (a.dh0) k_no_steps<<<blocks(n), kLanes, 0, s>>>(a.dh_last, a.dh0, n);
    if (a.dbias) k_no_steps<<<blocks(nb), kLanes, 0, s>>>(nullptr, a.dbias, nb);
    return hipGetLastError();
  }
  k_backward_chunks<E><<<dim3(blocks(n), chunks), kLanes, 0, s>>>(a, chunks);
  k_backward_carry<<<blocks(n), kLanes, 0, s>>>(a, chunks);
  k_backward<E><<<dim3(blocks(n), chunks), kLanes, 0, s>>>(a, chunks);
  if (a.dbias) k_bias_sum<<<blocks(nb), kLanes, 0, s>>>(a.ws + n * chunks, a.dbias, nb, a.C, (int64_t)a.B * chunks);
  return hipGetLastError();
}

template <typename E> hipError_t step(const RecurArgs& a, hipStream_t s) {
  k_step<E><<<blocks((int64_t)a.P * a.B * a.C), kLanes, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace recur
}  // namespace

int64_t recur_workspace_floats(int64_t P, int64_t B, int64_t T, int64_t C) { return 3 * P * B * recur_chunks(T) * C; }

hipError_t launch_recur_forward(const RecurArgs& a, int dtype, hipStream_t s) {
  return dtype == POP_F32 ? recur::forward<float>(a, s) : dtype == POP_BF16 ? recur::forward<__bf16>(a, s) : recur::forward<_Float16>(a, s);
}
hipError_t launch_recur_backward(const RecurArgs& a, int dtype, hipStream_t s) {
  return dtype == POP_F32 ? recur::backward<float>(a, s) : dtype == POP_BF16 ? recur::backward<__bf16>(a, s) : recur::backward<_Float16>(a, s);
}
hipError_t launch_recur_step(const RecurArgs& a, int dtype, hipStream_t s) {
  return dtype == POP_F32 ? recur::step<float>(a, s) : dtype == POP_BF16 ? recur::step<__bf16>(a, s) : recur::step<_Float16>(a, s);
}

}  // namespace pop
