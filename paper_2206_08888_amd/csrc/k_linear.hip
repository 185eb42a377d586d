// Linear attention with a decay for each head over sequences, its backward pass, and single steps (operators.h).
//
// Step by step: a workgroup per agent, sequence and head holds its state in registers.
#include <hip/hip_runtime.h>
#include "operators.h"

namespace pop {
namespace {
namespace linear {

constexpr int kThreads = 256, kMost = POP_LINEAR_MAX_DIM;

__device__ inline float log_decay_of(const float* log_decay, int at) { return log_decay ? fminf(fmaxf(log_decay[at], -200.0f), 0.0f) : 0.0f; }
template <typename E> __device__ inline const E* at(const pop_heads& s, int p, int b, int h) { return (const E*)s.data + p * s.agent + b * s.row + h * s.head; }

// Thread t has column t % width of the state, rows t / width + i * groups.
template <typename E> __global__ void __launch_bounds__(kThreads) k_rows(LinearArgs a) {
  __shared__ float sq[kMost], sk[kMost], part[kThreads];
  const LinearRole& r = a.role[blockIdx.y];
  const int col = blockIdx.x, h = col % a.H, row = col / a.H, b = row % a.B, p = row / a.B;
  const int len = a.lengths ? min(max(a.lengths[row], 0), a.T) : a.T;
  const float lambda = expf(log_decay_of(a.log_decay, p * a.H + h));
  const uint8_t* reset = (const uint8_t*)a.reset.data;
  if (reset) reset += p * a.reset.agent + b * a.reset.row;
  int width = 1;
  while (width < r.V) width *= 2;
  const int groups = kThreads / width, j = threadIdx.x % width, g = threadIdx.x / width;
  const bool on = j < r.V;
  float S[kMost / 2];
  const int64_t state = (int64_t)col * r.K * r.V;
#pragma unroll
  for (int i = 0; i < kMost / 2; ++i) {
    const int k = g + i * groups;
    S[i] = on && k < r.K && r.first ? r.first[state + k * r.first_k + j * r.first_v] : 0.0f;
  }
  for (int n = 0; n < len; ++n) {
    const int t = r.reverse ? len - 1 - n : n;
    for (int i = threadIdx.x; i < r.K; i += kThreads) {
      sq[i] = (float)at<E>(r.q, p, b, h)[t * r.q.step + i];
      sk[i] = (float)at<E>(r.k, p, b, h)[t * r.k.step + i] * r.write;
    }
    const float v = on ? (float)at<E>(r.v, p, b, h)[t * r.v.step + j] : 0.0f;
    const bool cut = reset && (r.reverse ? t + 1 < len && reset[(t + 1) * a.reset.step] : reset[t * a.reset.step]);
    const float f = r.reverse && n == 0 ? 1.0f : lambda;
    __syncthreads();
    float o = 0.0f;
#pragma unroll
    for (int i = 0; i < kMost / 2; ++i) {
      const int k = g + i * groups;
      if (k >= r.K) break;
      S[i] = fmaf(sk[k], v, cut ? 0.0f : f * S[i]);
      o = fmaf(sq[k], S[i], o);
    }
    part[threadIdx.x] = o;
    __syncthreads();
    if (g == 0 && on) {
      for (int i = 1; i < groups; ++i) o += part[i * width + j];
      ((E*)r.o.data)[p * r.o.agent + b * r.o.row + h * r.o.head + t * r.o.step + j] = (E)(o * r.read);
    }
  }
  if (g == 0 && on)
    for (int t = len; t < a.T; ++t) ((E*)r.o.data)[p * r.o.agent + b * r.o.row + h * r.o.head + t * r.o.step + j] = (E)0.0f;
  if (!r.last) return;
  const bool cut = r.reverse && len > 0 && reset && reset[0];
  const float f = r.reverse && len > 0 ? lambda : 1.0f;
#pragma unroll
  for (int i = 0; i < kMost / 2; ++i) {
    const int k = g + i * groups;
    if (on && k < r.K) r.last[state + k * r.V + j] = cut ? 0.0f : f * S[i];
  }
}

template <typename E> __global__ void __launch_bounds__(kThreads) k_step(LinearStep a) {
  __shared__ float sq[kMost], sk[kMost], part[kThreads];
  const int h = blockIdx.x % a.H, row = blockIdx.x / a.H, b = row % a.B, p = row / a.B;
  const int slot = a.slots ? a.slots[row] : b;
  E* o = (E*)a.o.data + p * a.o.agent + b * a.o.row + h * a.o.head;
  if (slot < 0 || slot >= a.n_slots) {
    for (int i = threadIdx.x; i < a.V; i += kThreads) o[i] = (E)0.0f;
    return;
  }
  for (int i = threadIdx.x; i < a.K; i += kThreads) {
    sq[i] = (float)at<E>(a.q, p, b, h)[i];
    sk[i] = (float)at<E>(a.k, p, b, h)[i];
  }
  const bool cut = a.reset.data && ((const uint8_t*)a.reset.data)[p * a.reset.agent + b * a.reset.row];
  const float lambda = expf(log_decay_of(a.log_decay, p * a.H + h));
  int width = 1;
  while (width < a.V) width *= 2;
  const int groups = kThreads / width, j = threadIdx.x % width, g = threadIdx.x / width;
  float* S = a.state + (((int64_t)p * a.n_slots + slot) * a.H + h) * a.K * a.V;
  __syncthreads();
  float sum = 0.0f;
  if (j < a.V) {
    const float v = (float)at<E>(a.v, p, b, h)[j];
    for (int k = g; k < a.K; k += groups) {
      const float s = fmaf(sk[k], v, cut ? 0.0f : lambda * S[k * a.V + j]);
      S[k * a.V + j] = s;
      sum = fmaf(sq[k], s, sum);
    }
  }
  part[threadIdx.x] = sum;
  __syncthreads();
  if (g == 0 && j < a.V) {
    for (int i = 1; i < groups; ++i) sum += part[i * width + j];
    o[j] = (E)(sum * a.scale);
  }
}

template <typename E> hipError_t run(const LinearArgs& a, hipStream_t s) {
  k_rows<E><<<dim3((unsigned)(a.P * a.B * a.H), a.roles), kThreads, 0, s>>>(a);
  return hipGetLastError();
}
template <typename E> hipError_t step(const LinearStep& a, hipStream_t s) {
  k_step<E><<<(unsigned)(a.P * a.B * a.H), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace linear
}  // namespace

int64_t linear_workspace_bytes(int64_t P, int64_t B, int64_t T, int64_t H, int64_t K, int64_t V, int64_t element, bool backward) { return 0; }

hipError_t launch_linear(const LinearArgs& a, int dtype, void* ws, hipStream_t s) {
  return dtype == POP_F32 ? linear::run<float>(a, s) : dtype == POP_BF16 ? linear::run<__bf16>(a, s) : linear::run<_Float16>(a, s);
}
hipError_t launch_linear_step(const LinearStep& a, int dtype, hipStream_t s) {
  return dtype == POP_F32 ? linear::step<float>(a, s) : dtype == POP_BF16 ? linear::step<__bf16>(a, s) : linear::step<_Float16>(a, s);
}

}  // namespace pop
