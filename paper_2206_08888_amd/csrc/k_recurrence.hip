// Gated linear recurrence over sequences, its backward pass, and single steps (operators.h).
//
//   a_t = sigmoid(g_t + bias),  h_t = a_t keep_t h_{t-1} + (1 - a_t) x_t;  keep_t = 0 at resets
//   backward, d_t = dL/dh_t:  d_t = dy_t + a_{t+1} keep_{t+1} d_{t+1};  dx_t = d_t (1 - a_t);
//   dg_t = d_t (keep_t h_{t-1} - x_t) a_t (1 - a_t);  dbias = sum dg;  dh0 = a_0 keep_0 d_0
//
// Both directions are scans: a run of steps maps the state s in front of it (backward: the gradient behind it) to
// A s + H with A the product of its a keep, and such maps compose.  A run with a reset has A = -0: then s is left out,
// not multiplied (it may be NaN or infinite).
//
// The columns of a call are its P * batch * C channels.  A workgroup takes 64 of them through tiles of kRecurChunk =
// 128 steps.  A lane holds 32 elements of a tile in registers, V adjacent channels x K = 32 / V successive steps, finds
// the map of its steps, one wavefront (a column per lane) carries the state over the tile's runs, and the lanes go over
// their steps again from the state in front of them: every element is read once and its gate computed once.
#include <hip/hip_runtime.h>
#include "operators.h"

namespace pop {
namespace {
namespace recur {

constexpr int kThreads = 256, kColumns = 64;

// sigmoid(z) and 1 - sigmoid(z), each to fp32's precision
struct Gate { float a, b; };
__device__ inline Gate gate(float z) {
  const float e = __expf(-fabsf(z)), big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  return z >= 0.0f ? Gate{big, small} : Gate{small, big};                     // NaN: e is NaN, and so are both
}

__device__ inline bool cut(float A) { return __float_as_uint(A) >> 31; }                    // the run has a reset
__device__ inline float apply(float A, float H, float s) { return cut(A) ? H : fmaf(A, s, H); }
__device__ inline float compose(float A, float B) { return cut(A) || cut(B) ? -0.0f : A * B; }

// What waits for LDS only: loads of the next tile stay in flight across it.
__device__ inline void sync_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <typename E, int V> struct Shape {
  typedef E vec __attribute__((ext_vector_type(V)));
  static constexpr int K = 32 / V, kLanes = kColumns / V, kRuns = kThreads / kLanes;
  static_assert(kRuns * K == kRecurChunk, "a tile is a chunk");
};
template <typename E> struct Shape<E, 1> {
  typedef E vec;
  static constexpr int K = 32, kLanes = kColumns, kRuns = kThreads / kLanes;
};
template <int V, typename T> __device__ inline float element(const T& v, int i) {
  if constexpr (V == 1) return (float)v; else return (float)v[i];
}

// The columns of a lane: `c` and the V - 1 behind it, of one sequence.
struct Lane {
  bool on;
  int c, p, b, row, len;
};
__device__ inline Lane lane_at(const RecurArgs& a, int64_t column) {
  Lane l;
  l.on = column < (int64_t)a.P * a.B * a.C;
  const int i = l.on ? (int)column : 0;
  l.row = i / a.C;
  l.c = i - l.row * a.C;
  l.p = l.row / a.B;
  l.b = l.row - l.p * a.B;
  l.len = !l.on ? 0 : a.lengths ? min(max(a.lengths[l.row], 0), a.T) : a.T;
  return l;
}
__device__ inline int64_t base(const pop_sequence& s, const Lane& l) { return l.p * s.agent + l.b * s.row; }

// K steps of a lane's columns of one array, from step t on; steps at or behind `end` are not read (and stay as they are).
template <typename E, int V> struct Strip {
  typename Shape<E, V>::vec v[Shape<E, V>::K];
  __device__ inline void load(const pop_sequence& s, const Lane& l, int t, int end, bool whole) {
    const E* p = (const E*)s.data + base(s, l) + l.c + (int64_t)t * s.step;
    if (whole) {
#pragma unroll
      for (int k = 0; k < Shape<E, V>::K; ++k) v[k] = *(const typename Shape<E, V>::vec*)(p + k * s.step);
    } else {
#pragma unroll
      for (int k = 0; k < Shape<E, V>::K; ++k)
        if (t + k < end) v[k] = *(const typename Shape<E, V>::vec*)(p + k * s.step);
    }
  }
};

template <typename E, int V>
__device__ inline void store(const pop_sequence& s, const Lane& l, int t, const float (&v)[V]) {
  typename Shape<E, V>::vec o;
  if constexpr (V == 1) {
    o = (E)v[0];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = (E)v[i];
  }
  *(typename Shape<E, V>::vec*)((E*)s.data + base(s, l) + l.c + (int64_t)t * s.step) = o;
}

// Bit k: step t + k starts an episode.
template <int K> __device__ inline unsigned resets(const RecurArgs& a, const Lane& l, int t) {
  unsigned m = 0;
  if (a.reset.data) {
    const uint8_t* r = (const uint8_t*)a.reset.data + base(a.reset, l) + (int64_t)t * a.reset.step;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (t + k < l.len) m |= (r[k * a.reset.step] != 0 ? 1u : 0u) << k;
  }
  return m;
}

// ---- forward

// kWhole: a workgroup goes through whole sequences.  Otherwise sequences are cut into segments of `per` chunks: kMaps
// finds each segment's map, kSegments starts every segment from the maps in front of it.
enum { kWhole = 0, kMaps = 1, kSegments = 2 };

// The state at the start of segment `seg` (direction 1: behind it, coming from the end) of this lane's column, wavefront
// 0's result; all four wavefronts compose a quarter of the maps each.
__device__ inline float enter(const RecurArgs& a, int64_t n, int64_t column, int from, int count, int stride, float s, float (*quarter)[2][kColumns]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, q = (count + 3) / 4;
  const int lo = min(wave * q, count), hi = min(lo + q, count);
  float A = 1.0f, H = 0.0f;
  if (column < n) {
    const float* at = a.ws + (int64_t)(from + lo * stride) * n + column;
    const int64_t segments = (int64_t)gridDim.y * n;
#pragma unroll 8
    for (int i = lo; i < hi; ++i, at += stride * n) {
      H = apply(at[0], at[segments], H);
      A = compose(A, at[0]);
    }
  }
  quarter[wave][0][lane] = A;
  quarter[wave][1][lane] = H;
  sync_lds();
#pragma unroll
  for (int w = 0; w < 4; ++w) s = apply(quarter[w][0][lane], quarter[w][1][lane], s);
  return s;
}

template <typename E, int V, int MODE>
__global__ void __launch_bounds__(kThreads) k_forward(RecurArgs a, int chunks, int per) {
  using S = Shape<E, V>;
  __shared__ float runs[2][2][S::kRuns][kColumns];             // [tile parity][A, H or the state in front][run][column]
  __shared__ float quarter[4][2][kColumns];
  const int64_t n = (int64_t)a.P * a.B * a.C, first = (int64_t)blockIdx.x * kColumns;
  const int at = threadIdx.x % S::kLanes, run = threadIdx.x / S::kLanes;
  const Lane l = lane_at(a, first + at * V);
  const int k0 = blockIdx.y * per, k1 = min(k0 + per, chunks);
  float bias[V];
#pragma unroll
  for (int v = 0; v < V; ++v) bias[v] = a.bias && l.on ? a.bias[(int64_t)l.p * a.C + l.c + v] : 0.0f;

  Strip<E, V> x, g;
  unsigned mask;
  const auto fetch = [&](int k) {
    const int t = k * kRecurChunk + run * S::K;
    const bool whole = __all(t + S::K <= l.len);
    x.load(a.x, l, t, l.len, whole);
    g.load(a.g, l, t, l.len, whole);
    mask = resets<S::K>(a, l, t);
  };
  fetch(k0);

  // wavefront 0: a column per lane
  const int64_t column = first + threadIdx.x;
  float carry = 0.0f, A_all = 1.0f;
  if (MODE != kMaps) {
    const int64_t col = first + (threadIdx.x & 63);
    if (a.h0 && col < n) carry = a.h0[col];
    if (MODE == kSegments) carry = enter(a, n, col, 0, blockIdx.y, 1, carry, quarter);
  }

  for (int k = k0; k < k1; ++k) {
    const int t = k * kRecurChunk + run * S::K;
    float A[V], H[V], m[S::K][V], u[S::K][V];                  // the run's map, multipliers and inputs of its steps
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
#pragma unroll
    for (int i = 0; i < S::K; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gate q = gate(element<V>(g.v[i], v) + bias[v]);
        const bool live = t + i < l.len;
        m[i][v] = live ? q.a : 1.0f;
        u[i][v] = live ? q.b * element<V>(x.v[i], v) : 0.0f;
      }
    const unsigned here = mask;
    const bool any = __any(here != 0);
    if (any) {
#pragma unroll
      for (int i = 0; i < S::K; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const bool r = here >> i & 1;
          H[v] = r ? u[i][v] : fmaf(m[i][v], H[v], u[i][v]);
          A[v] = A[v] * m[i][v];
        }
#pragma unroll
      for (int v = 0; v < V; ++v) A[v] = here ? -0.0f : A[v];
    } else {
#pragma unroll
      for (int i = 0; i < S::K; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          H[v] = fmaf(m[i][v], H[v], u[i][v]);
          A[v] = A[v] * m[i][v];
        }
    }
    if (k + 1 < k1) fetch(k + 1);
    auto& sA = runs[k & 1][0];
    auto& sH = runs[k & 1][1];
#pragma unroll
    for (int v = 0; v < V; ++v) { sA[run][at * V + v] = A[v]; sH[run][at * V + v] = H[v]; }
    sync_lds();
    if (threadIdx.x < kColumns) {
      if (MODE != kMaps && a.states && column < n) {
        const int64_t row = column / a.C;
        a.states[(row * chunks + k) * a.C + (column - row * a.C)] = carry;
      }
#pragma unroll
      for (int i = 0; i < S::kRuns; ++i) {
        const float Ai = sA[i][threadIdx.x], Hi = sH[i][threadIdx.x];
        if (MODE == kMaps) A_all = compose(A_all, Ai);
        else sH[i][threadIdx.x] = carry;
        carry = apply(Ai, Hi, carry);
      }
    }
    if (MODE == kMaps) continue;                               // the next tile has the other half of `runs`
    sync_lds();
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = sH[run][at * V + v];
    const bool inside = __all(l.on && t + S::K <= a.T), full = __all(t + S::K <= l.len);
#pragma unroll
    for (int i = 0; i < S::K; ++i) {
      float y[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (any) h[v] = here >> i & 1 ? u[i][v] : fmaf(m[i][v], h[v], u[i][v]);
        else h[v] = fmaf(m[i][v], h[v], u[i][v]);
        y[v] = full || t + i < l.len ? h[v] : 0.0f;
      }
      if (inside || (l.on && t + i < a.T)) store<E, V>(a.y, l, t + i, y);
    }
  }
  if (threadIdx.x < kColumns && column < n) {
    if (MODE == kMaps) {
      float* to = a.ws + (int64_t)blockIdx.y * n + column;
      to[0] = A_all;
      to[(int64_t)gridDim.y * n] = carry;
    } else if (a.h_last && k1 == chunks) {
      a.h_last[column] = carry;
    }
  }
}

__global__ void __launch_bounds__(kThreads) k_no_steps(const float* from, float* to, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) to[i] = from ? from[i] : 0.0f;
}

// ---- backward

// A segment's map of the gradient behind it to the one in front of it.
template <typename E, int V>
__global__ void __launch_bounds__(kThreads) k_backward_maps(RecurArgs a, int chunks, int per) {
  using S = Shape<E, V>;
  __shared__ float runs[2][2][S::kRuns][kColumns];
  const int64_t n = (int64_t)a.P * a.B * a.C, first = (int64_t)blockIdx.x * kColumns, column = first + threadIdx.x;
  const int at = threadIdx.x % S::kLanes, run = threadIdx.x / S::kLanes;
  const Lane l = lane_at(a, first + at * V);
  const int k0 = blockIdx.y * per, k1 = min(k0 + per, chunks);
  float bias[V];
#pragma unroll
  for (int v = 0; v < V; ++v) bias[v] = a.bias && l.on ? a.bias[(int64_t)l.p * a.C + l.c + v] : 0.0f;
  Strip<E, V> g, dy;
  unsigned mask;
  const auto fetch = [&](int k) {
    const int t = k * kRecurChunk + run * S::K;
    const bool whole = __all(t + S::K <= l.len);
    g.load(a.g, l, t, l.len, whole);
    dy.load(a.dy, l, t, l.len, whole);
    mask = resets<S::K>(a, l, t);
  };
  fetch(k1 - 1);
  float d = 0.0f, A_all = 1.0f;
  for (int k = k1 - 1; k >= k0; --k) {
    const int t = k * kRecurChunk + run * S::K;
    float A[V], D[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; D[v] = 0.0f; }
#pragma unroll
    for (int i = S::K - 1; i >= 0; --i)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float q = gate(element<V>(g.v[i], v) + bias[v]).a;
        if (t + i < l.len) {
          D[v] = mask >> i & 1 ? 0.0f : q * (D[v] + element<V>(dy.v[i], v));
          A[v] *= q;
        }
      }
    const unsigned here = mask;
    if (k > k0) fetch(k - 1);
    auto& sA = runs[k & 1][0];
    auto& sD = runs[k & 1][1];
#pragma unroll
    for (int v = 0; v < V; ++v) { sA[run][at * V + v] = here ? -0.0f : A[v]; sD[run][at * V + v] = D[v]; }
    sync_lds();
    if (threadIdx.x < kColumns) {
#pragma unroll
      for (int i = S::kRuns - 1; i >= 0; --i) {
        const float Ai = sA[i][threadIdx.x];
        A_all = compose(A_all, Ai);
        d = apply(Ai, sD[i][threadIdx.x], d);
      }
    }
  }
  if (threadIdx.x < kColumns && column < n) {
    float* to = a.ws + (int64_t)blockIdx.y * n + column;
    to[0] = A_all;
    to[(int64_t)gridDim.y * n] = d;
  }
}

// dx and dg, and the sums of dg over the segment to `sums` [segments, columns].
template <typename E, int V>
__global__ void __launch_bounds__(kThreads) k_backward(RecurArgs a, int chunks, int per, float* sums) {
  using S = Shape<E, V>;
  __shared__ float runs[2][3][S::kRuns][kColumns];             // [tile parity][A; H, then states in front; D, then gradients behind]
  __shared__ float quarter[4][2][kColumns];
  const int64_t n = (int64_t)a.P * a.B * a.C, first = (int64_t)blockIdx.x * kColumns;
  const int at = threadIdx.x % S::kLanes, run = threadIdx.x / S::kLanes, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Lane l = lane_at(a, first + at * V);
  const int k0 = blockIdx.y * per, k1 = min(k0 + per, chunks);
  float bias[V];
#pragma unroll
  for (int v = 0; v < V; ++v) bias[v] = a.bias && l.on ? a.bias[(int64_t)l.p * a.C + l.c + v] : 0.0f;
  Strip<E, V> x, g, dy;
  unsigned mask;
  const auto fetch = [&](int k) {
    const int t = k * kRecurChunk + run * S::K;
    const bool whole = __all(t + S::K <= l.len);
    x.load(a.x, l, t, l.len, whole);
    g.load(a.g, l, t, l.len, whole);
    dy.load(a.dy, l, t, l.len, whole);
    mask = resets<S::K>(a, l, t);
  };
  fetch(k1 - 1);
  // a column per lane: wavefront 0 carries the gradient from tile to tile, wavefront 1 takes states from `states`
  const int64_t column = first + lane, row = column / a.C;
  const bool valid = column < n;
  float d = a.dh_last && valid ? a.dh_last[column] : 0.0f;
  if (gridDim.y > 1) d = enter(a, n, column, gridDim.y - 1, gridDim.y - 1 - blockIdx.y, -1, d, quarter);
  const float* states = a.states + row * chunks * a.C + (column - row * a.C);
  float sum[V];
#pragma unroll
  for (int v = 0; v < V; ++v) sum[v] = 0.0f;

  for (int k = k1 - 1; k >= k0; --k) {
    const int t = k * kRecurChunk + run * S::K;
    const unsigned here = mask;
    const float state = wave == 1 && valid ? states[(int64_t)k * a.C] : 0.0f;
    float A[V], H[V], D[V], ga[S::K][V], gb[S::K][V], xs[S::K][V], ds[S::K][V];
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = D[v] = 0.0f; }
#pragma unroll
    for (int i = 0; i < S::K; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gate q = gate(element<V>(g.v[i], v) + bias[v]);
        const bool live = t + i < l.len;
        ga[i][v] = live ? q.a : 1.0f;
        gb[i][v] = live ? q.b : 0.0f;
        xs[i][v] = live ? element<V>(x.v[i], v) : 0.0f;
        ds[i][v] = live ? element<V>(dy.v[i], v) : 0.0f;
        const float u = gb[i][v] * xs[i][v];
        H[v] = here >> i & 1 ? u : fmaf(ga[i][v], H[v], u);
        A[v] *= ga[i][v];
      }
#pragma unroll
    for (int i = S::K - 1; i >= 0; --i)
#pragma unroll
      for (int v = 0; v < V; ++v) D[v] = here >> i & 1 ? 0.0f : ga[i][v] * (D[v] + ds[i][v]);
    if (k > k0) fetch(k - 1);
    auto& sA = runs[k & 1][0];
    auto& sH = runs[k & 1][1];
    auto& sD = runs[k & 1][2];
#pragma unroll
    for (int v = 0; v < V; ++v) { sA[run][at * V + v] = here ? -0.0f : A[v]; sH[run][at * V + v] = H[v]; sD[run][at * V + v] = D[v]; }
    sync_lds();
    if (wave == 0) {
#pragma unroll
      for (int i = S::kRuns - 1; i >= 0; --i) {
        const float Ai = sA[i][lane], Di = sD[i][lane];
        sD[i][lane] = d;
        d = apply(Ai, Di, d);
      }
    } else if (wave == 1) {
      float s = state;
#pragma unroll
      for (int i = 0; i < S::kRuns; ++i) {
        const float Ai = sA[i][lane], Hi = sH[i][lane];
        sH[i][lane] = s;
        s = apply(Ai, Hi, s);
      }
    }
    sync_lds();
    float h[V], e[V], before[S::K][V];
#pragma unroll
    for (int v = 0; v < V; ++v) { h[v] = sH[run][at * V + v]; e[v] = sD[run][at * V + v]; }
#pragma unroll
    for (int i = 0; i < S::K; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        before[i][v] = here >> i & 1 ? 0.0f : h[v];
        h[v] = here >> i & 1 ? gb[i][v] * xs[i][v] : fmaf(ga[i][v], h[v], gb[i][v] * xs[i][v]);
      }
    const bool inside = __all(l.on && t + S::K <= a.T);
#pragma unroll
    for (int i = S::K - 1; i >= 0; --i) {
      float dx[V], dg[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const bool live = t + i < l.len;
        const float at_t = e[v] + ds[i][v];
        dx[v] = live ? at_t * gb[i][v] : 0.0f;
        dg[v] = live ? at_t * (before[i][v] - xs[i][v]) * (ga[i][v] * gb[i][v]) : 0.0f;
        sum[v] += dg[v];
        e[v] = here >> i & 1 ? 0.0f : ga[i][v] * at_t;
      }
      if (inside || (l.on && t + i < a.T)) {
        store<E, V>(a.dx, l, t + i, dx);
        store<E, V>(a.dg, l, t + i, dg);
      }
    }
  }
  if (a.dh0 && k0 == 0 && wave == 0 && valid) a.dh0[column] = d;
  if (!a.dbias) return;
  sync_lds();                                                  // the last tile's states are read
  auto& part = runs[0][0];
#pragma unroll
  for (int v = 0; v < V; ++v) part[run][at * V + v] = sum[v];
  sync_lds();
  if (wave == 0 && valid) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i) s += part[i][lane];
    sums[(int64_t)blockIdx.y * n + column] = s;
  }
}

// dbias from the sums of every segment and sequence
__global__ void __launch_bounds__(kThreads) k_bias_sum(const float* sums, float* dbias, int P, int B, int C, int segments) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, n = (int64_t)P * B * C;
  if (i >= (int64_t)P * C) return;
  const int p = (int)(i / C), c = (int)(i % C);
  float v = 0.0f;
  for (int s = 0; s < segments; ++s) {
    const float* at = sums + s * n + (int64_t)p * B * C + c;
#pragma unroll 8
    for (int b = 0; b < B; ++b) v += at[(int64_t)b * C];
  }
  dbias[i] = v;
}

// ---- single steps

template <typename E>
__global__ void __launch_bounds__(kThreads) k_step(RecurArgs a) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const Lane l = lane_at(a, i);
  if (!l.on) return;
  const int slot = a.slots ? a.slots[l.row] : l.b;
  float h = 0.0f;
  if (slot >= 0 && slot < a.n_slots) {
    float* state = a.state + ((int64_t)l.p * a.n_slots + slot) * a.C + l.c;
    const Gate q = gate((float)((const E*)a.g.data)[base(a.g, l) + l.c] + (a.bias ? a.bias[(int64_t)l.p * a.C + l.c] : 0.0f));
    const float u = q.b * (float)((const E*)a.x.data)[base(a.x, l) + l.c];
    const bool r = a.reset.data && ((const uint8_t*)a.reset.data)[base(a.reset, l)] != 0;
    h = r ? u : fmaf(q.a, *state, u);
    *state = h;
  }
  ((E*)a.y.data)[base(a.y, l) + l.c] = (E)h;
}

// ---- launches

unsigned blocks(int64_t n) { return (unsigned)((n + kThreads - 1) / kThreads); }

// Sequences are cut where their columns alone do not fill the chip.
struct Cut { int chunks, per, segments; };
constexpr int kMaxSegments = 128;
Cut cut_of(int64_t P, int64_t B, int64_t T, int64_t C) {
  const int64_t groups = (P * B * C + kColumns - 1) / kColumns, chunks = recur_chunks(T);
  int64_t want = groups >= 512 ? 1 : (1024 + groups - 1) / groups;
  if (want > kMaxSegments) want = kMaxSegments;
  if (want > chunks) want = chunks;
  const int64_t per = (chunks + want - 1) / want;
  return {(int)chunks, (int)per, (int)((chunks + per - 1) / per)};
}

// Whether every row of an array can be read in vectors of 4 elements.
bool wide(const pop_sequence& s, int64_t bytes) {
  return (uintptr_t)s.data % (4 * bytes) == 0 && s.agent % 4 == 0 && s.row % 4 == 0 && s.step % 4 == 0;
}

template <typename E, int V> void forward(const RecurArgs& a, const Cut& c, dim3 grid, hipStream_t s) {
  if (c.segments == 1) {
    k_forward<E, V, kWhole><<<grid, kThreads, 0, s>>>(a, c.chunks, c.per);
  } else {
    k_forward<E, V, kMaps><<<grid, kThreads, 0, s>>>(a, c.chunks, c.per);
    k_forward<E, V, kSegments><<<grid, kThreads, 0, s>>>(a, c.chunks, c.per);
  }
}
template <typename E> hipError_t forward(const RecurArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.P * a.B * a.C;
  if (a.T == 0) {
    if (a.h_last) k_no_steps<<<blocks(n), kThreads, 0, s>>>(a.h0, a.h_last, n);
    return hipGetLastError();
  }
  const Cut c = cut_of(a.P, a.B, a.T, a.C);
  const dim3 grid((unsigned)((n + kColumns - 1) / kColumns), c.segments);
  const int64_t e = sizeof(E);
  if (a.C % 4 == 0 && wide(a.x, e) && wide(a.g, e) && wide(a.y, e)) forward<E, 4>(a, c, grid, s);
  else forward<E, 1>(a, c, grid, s);
  return hipGetLastError();
}

template <typename E, int V> void backward(const RecurArgs& a, const Cut& c, dim3 grid, float* sums, hipStream_t s) {
  if (c.segments > 1) k_backward_maps<E, V><<<grid, kThreads, 0, s>>>(a, c.chunks, c.per);
  k_backward<E, V><<<grid, kThreads, 0, s>>>(a, c.chunks, c.per, sums);
}
template <typename E> hipError_t backward(const RecurArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.P * a.B * a.C, nb = (int64_t)a.P * a.C;
  if (a.T == 0) {
    if (a.dh0) k_no_steps<<<blocks(n), kThreads, 0, s>>>(a.dh_last, a.dh0, n);
    if (a.dbias) k_no_steps<<<blocks(nb), kThreads, 0, s>>>(nullptr, a.dbias, nb);
    return hipGetLastError();
  }
  const Cut c = cut_of(a.P, a.B, a.T, a.C);
  const dim3 grid((unsigned)((n + kColumns - 1) / kColumns), c.segments);
  const int64_t e = sizeof(E);
  float* sums = a.ws + 2 * n * c.segments;
  if (a.C % 4 == 0 && wide(a.x, e) && wide(a.g, e) && wide(a.dy, e) && wide(a.dx, e) && wide(a.dg, e)) backward<E, 4>(a, c, grid, sums, s);
  else backward<E, 1>(a, c, grid, sums, s);
  if (a.dbias) k_bias_sum<<<blocks(nb), kThreads, 0, s>>>(sums, a.dbias, a.P, a.B, a.C, c.segments);
  return hipGetLastError();
}

template <typename E> hipError_t step(const RecurArgs& a, hipStream_t s) {
  k_step<E><<<blocks((int64_t)a.P * a.B * a.C), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace recur
}  // namespace

int64_t recur_workspace_floats(int64_t P, int64_t B, int64_t T, int64_t C) { return T == 0 ? 0 : 3 * P * B * C * recur::cut_of(P, B, T, C).segments; }

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
