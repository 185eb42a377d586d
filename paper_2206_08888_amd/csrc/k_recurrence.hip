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
// their steps again from the state in front of them: every element is read once and its gate computed once.  Wavefronts
// whose steps all exist and have no resets among them skip what is for those.
//
// Where the columns do not fill the chip, sequences are shared by several workgroups: each tile has a workgroup of its own
// that waits for the state of the one before (kChain), or, where columns are so few that this wait would be the longest part,
// sequences are cut into segments whose maps a launch of its own finds (kMaps, kSegments), at the price of reading x and g
// twice.
#include <hip/hip_runtime.h>
#include "operators.h"

namespace pop {
namespace {
namespace recur {

constexpr int kThreads = 256, kColumns = 64;

// a = sigmoid(z) and b = 1 - sigmoid(z).  The sum z = g + bias is rounded before the factor log2 e, which is no more than its own
// rounding; with the factor on both parts, one fused product, gates whose parts cancel lose it (at a bias of 100, relative
// errors of 5e-6).  The reciprocal is off by up to a unit: in fp32 the larger of the two comes as 1 minus the smaller,
// right to half a unit, as states and gradients pass through hundreds of gates near one (23 agents of 3 x 777 x 129, error of dh0
// 1.4e-7 against 3.1e-7; the same time).  For 16-bit arrays, whose own rounding of g is 2^-9 or 2^-12 of it, that is left out:
// 80 agents of 8 x 512 x 256, forward and backward, 325 us with it, 315 without.
struct Gate { float a, b; };
constexpr float kLog2e = 1.44269504f;
template <typename E> __device__ inline Gate gate(float z) {
  const float t = -kLog2e * z;
  const float e = __builtin_amdgcn_exp2f(t), r = __builtin_amdgcn_rcpf(1.0f + e);
  const bool up = t > 0.0f;                                   // then r <= 1/2, and e may be infinite
  if constexpr (sizeof(E) == 4) {
    const float small = up ? r : e * r, large = 1.0f - small;
    return {up ? small : large, up ? large : small};
  }
  return {r, up ? 1.0f - r : e * r};
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

// V adjacent channels of a lane, N elements of a tile.
template <typename E, int V> struct Vec { typedef E type __attribute__((ext_vector_type(V))); };
template <typename E> struct Vec<E, 1> { typedef E type; };
template <typename E, int V, int N> struct Shape {
  typedef typename Vec<E, V>::type vec;
  static constexpr int K = N / V, kLanes = kColumns / V, kRuns = kRecurChunk / K, kThreads = kLanes * kRuns;
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

// A lane's columns of one array, a step after the other: the offset is carried along (kept from being taken apart into
// K products of the stride, which do not fit the scalar registers).
#define POP_GLOBAL __attribute__((address_space(1)))
template <typename E, int V> struct Walk {
  typedef POP_GLOBAL typename Vec<E, V>::type* pointer;
  POP_GLOBAL char* start;
  int64_t at, step;                            // bytes
  __device__ inline Walk(const pop_sequence& s, int64_t element, int t)
      : start((POP_GLOBAL char*)s.data), at((element + (int64_t)t * s.step) * (int64_t)sizeof(E)), step(s.step * (int64_t)sizeof(E)) {}
  __device__ inline pointer p() const { return (pointer)(start + at); }
  __device__ inline void next(bool on = true) {
    at += on ? step : 0;
    asm("" : "+v"(at));
  }
};

// K steps of a lane's columns of one array from step t on.  Steps behind the array's end are read as its last one, steps
// behind the sequence's end as they are; neither is used.  (Loads under conditions of their own would each be waited for
// before the next: a wavefront reads all K steps, or, with every step behind its sequences' ends, none.)
template <typename E, int V, int K> struct Strip {
  typename Vec<E, V>::type v[K];
  __device__ inline void load(const pop_sequence& s, const Lane& l, int t, int T) {
    Walk<E, V> w(s, base(s, l) + l.c, min(t, T - 1));
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = *w.p();
      if (k + 1 < K) w.next(t + k + 1 < T);
    }
  }
};

template <typename E, int V>
__device__ inline void store(typename Walk<E, V>::pointer to, const float (&v)[V]) {
  typename Vec<E, V>::type o;
  if constexpr (V == 1) {
    o = (E)v[0];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = (E)v[i];
  }
  *to = o;
}

// Episode starts: bit k for step t + k.
template <int K> struct Resets {
  Strip<uint8_t, 1, K> r;
  __device__ inline void load(const RecurArgs& a, const Lane& l, int t) {
    if (!a.reset.data) return;
    Lane first = l;
    first.c = 0;
    r.load(a.reset, first, t, a.T);
  }
  __device__ inline unsigned bits(const RecurArgs& a, const Lane& l, int t) const {
    unsigned m = 0;
    if (a.reset.data)
#pragma unroll
      for (int k = 0; k < K; ++k) m |= (r.v[k] != 0 && t + k < l.len ? 1u : 0u) << k;
    return m;
  }
};

// ---- how sequences are shared

// kWhole: a workgroup goes through whole sequences.  kMaps finds the map of each segment of `per` tiles, kSegments starts
// every segment from the maps in front of it.  kChain: a tile per workgroup, which takes the state in front of it (the
// gradient behind it) from the workgroup before and hands its own on.
enum { kWhole = 0, kMaps = 1, kSegments = 2, kChain = 3 };

// Hand-over of kChain: a word per column and tile, the state with a 1 above it, written and read as one.  Words and the
// ticket behind them are cleared by a launch in front.  A workgroup's place in the chain goes by its ticket, not its
// index: the workgroup it waits for has an earlier ticket, so it runs or has ended, and by induction every wait ends.
__device__ inline unsigned long long* words_of(const RecurArgs& a) { return (unsigned long long*)a.ws; }
__device__ inline void hand_over(unsigned long long* word, float v) {
  __hip_atomic_store(word, 1ull << 32 | __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float taken_over(unsigned long long* word) {
  unsigned long long v;
  while (!((v = __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) >> 32)) __builtin_amdgcn_s_sleep(1);
  return __uint_as_float((unsigned)v);
}
__global__ void __launch_bounds__(kThreads) k_clear(unsigned long long* words, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) words[i] = 0;
}

// h0 (backward: dh_last) as the launch of maps found it, behind maps and sums: the last segment of kSegments writes
// h_last, which may lie over h0, while other segments have yet to start.  (kWhole reads and writes a column in one
// lane; in kChain only the first tile reads h0, and what the last one writes has passed through all of them.)
__device__ inline float* first_of(const RecurArgs& a, int64_t n, int segments) { return a.ws + 3 * n * segments + 2; }

// This workgroup's columns and tiles.
struct Place { int64_t first; int seg, segments; };
template <int MODE> __device__ inline Place place_of(const RecurArgs& a, int64_t n, int segments, bool backward) {
  if (MODE != kChain) return {(int64_t)blockIdx.x * kColumns, (int)blockIdx.y, segments};
  __shared__ unsigned ticket;
  if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add((unsigned*)(words_of(a) + (int64_t)segments * n), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  const unsigned groups = (unsigned)((n + kColumns - 1) / kColumns), t = ticket;
  const int seg = (int)(t / groups);
  return {(int64_t)(t % groups) * kColumns, backward ? segments - 1 - seg : seg, segments};
}

// The state at the start of segment `seg` (backward: the gradient behind it, from the end) of this lane's column; four
// wavefronts compose a quarter of the `count` maps each, from segment `from` on.
__device__ inline float enter(const RecurArgs& a, int64_t n, int64_t column, int segments, int from, int count, int stride, float s, float (*quarter)[2][kColumns]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, q = (count + 3) / 4;
  const int lo = min(wave * q, count), hi = min(lo + q, count);
  float A = 1.0f, H = 0.0f;
  if (wave < 4 && column < n) {
    const float* at = a.ws + (int64_t)(from + lo * stride) * n + column;
    const int64_t other = segments * n;
#pragma unroll 8
    for (int i = lo; i < hi; ++i, at += stride * n) {
      H = apply(at[0], at[other], H);
      A = compose(A, at[0]);
    }
  }
  if (wave < 4) {
    quarter[wave][0][lane] = A;
    quarter[wave][1][lane] = H;
  }
  sync_lds();
#pragma unroll
  for (int w = 0; w < 4; ++w) s = apply(quarter[w][0][lane], quarter[w][1][lane], s);
  return s;
}

template <int V> __device__ inline void bias_of(const RecurArgs& a, const Lane& l, float (&bias)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) bias[v] = a.bias && l.on ? a.bias[(int64_t)l.p * a.C + l.c + v] : 0.0f;
}

// ---- forward

// Bound by memory: x, g and y once, 3 elements a step and column.  kWhole, 80 agents of 8 x 512 steps x 256 columns in bf16:
// 122 us, 4.2 TB/s (a large copy: 4.8).  kChain, 10 agents of 4 x 1000 x 256 in fp32: 28 us, 4.3 TB/s, behind 3 of the
// clearing launch.  kMaps + kSegments, one sequence of 65536 x 256 in bf16: 16 + 25 us at 4.1 TB/s, two thirds of it x and g
// twice.  Single elements (V = 1, odd strides): 23 agents of 3 x 777 x 129 in fp32, half of the steps behind the ends: 24 us.
template <typename E, int V, int N, int MODE>
__global__ void __launch_bounds__(8192 / N) k_forward(RecurArgs a, int chunks, int per, int segments) {
  using S = Shape<E, V, N>;
  constexpr int K = S::K;
  __shared__ float runs[2][2][S::kRuns][kColumns];             // [tile parity][A, H or the state in front][run][column]
  __shared__ float quarter[4][2][kColumns];
  const int64_t n = (int64_t)a.P * a.B * a.C;
  const Place place = place_of<MODE>(a, n, segments, false);
  const int at = threadIdx.x % S::kLanes, run = threadIdx.x / S::kLanes;
  const Lane l = lane_at(a, place.first + at * V);
  const int k0 = place.seg * per, k1 = MODE == kChain ? k0 + 1 : min(k0 + per, chunks);
  float bias[V];
  bias_of<V>(a, l, bias);

  Strip<E, V, K> x, g;
  Resets<K> starts;
  const auto fetch = [&](int k) {
    const int t = k * kRecurChunk + run * K;
    if (!__any(t < l.len)) return;
    g.load(a.g, l, t, a.T);
    x.load(a.x, l, t, a.T);
    starts.load(a, l, t);
  };
  fetch(k0);

  // wavefront 0: a column per lane
  const int64_t column = place.first + (threadIdx.x & 63);
  const bool carries = threadIdx.x < kColumns && column < n;
  float carry = 0.0f, A_all = 1.0f;
  if (MODE == kMaps) {
    if (a.h0 && carries && place.seg == 0) first_of(a, n, segments)[column] = a.h0[column];
  } else {
    if (a.h0 && column < n && (MODE != kChain || place.seg == 0)) carry = MODE == kSegments ? first_of(a, n, segments)[column] : a.h0[column];
    if (MODE == kSegments) carry = enter(a, n, column, segments, 0, place.seg, 1, carry, quarter);
  }

  const int64_t row = column / a.C, y_at = base(a.y, l) + l.c;
  float* states = a.states + row * chunks * a.C + (column - row * a.C);

  for (int k = k0; k < k1; ++k) {
    const int t = k * kRecurChunk + run * K;
    float A[V], H[V], m[K][V], u[K][V];                        // the run's map, multipliers and inputs of its steps
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
    const unsigned here = starts.bits(a, l, t);
    const bool full = __all(t + K <= l.len), plain = full && !__any(here != 0);
    if (plain) {
#pragma unroll
      for (int i = 0; i < K; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const Gate q = gate<E>(element<V>(g.v[i], v) + bias[v]);
          m[i][v] = q.a;
          u[i][v] = q.b * element<V>(x.v[i], v);
          H[v] = fmaf(q.a, H[v], u[i][v]);
          A[v] *= q.a;
        }
    } else {
#pragma unroll
      for (int i = 0; i < K; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const Gate q = gate<E>(element<V>(g.v[i], v) + bias[v]);
          const bool live = t + i < l.len;
          m[i][v] = live ? q.a : 1.0f;
          u[i][v] = live ? q.b * element<V>(x.v[i], v) : 0.0f;
          H[v] = here >> i & 1 ? u[i][v] : fmaf(m[i][v], H[v], u[i][v]);
          A[v] *= m[i][v];
        }
#pragma unroll
      for (int v = 0; v < V; ++v) A[v] = here ? -0.0f : A[v];
    }
    if (MODE != kChain && k + 1 < k1) fetch(k + 1);
    auto& sA = runs[k & 1][0];
    auto& sH = runs[k & 1][1];
#pragma unroll
    for (int v = 0; v < V; ++v) { sA[run][at * V + v] = A[v]; sH[run][at * V + v] = H[v]; }
    sync_lds();
    if (threadIdx.x < kColumns) {
      if (MODE == kChain && place.seg > 0 && carries) carry = taken_over(words_of(a) + (int64_t)(place.seg - 1) * n + column);
      if (MODE != kMaps && a.states && carries) states[(int64_t)k * a.C] = carry;
#pragma unroll 8
      for (int i = 0; i < S::kRuns; ++i) {
        const float Ai = sA[i][threadIdx.x], Hi = sH[i][threadIdx.x];
        if (MODE == kMaps) A_all = compose(A_all, Ai);
        else sH[i][threadIdx.x] = carry;
        carry = apply(Ai, Hi, carry);
      }
      if (MODE == kChain && k1 < chunks && carries) hand_over(words_of(a) + (int64_t)place.seg * n + column, carry);
    }
    if (MODE == kMaps) continue;                               // the next tile has the other half of `runs`
    sync_lds();
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = sH[run][at * V + v];
    Walk<E, V> y(a.y, y_at, t);
    if (plain) {
#pragma unroll
      for (int i = 0; i < K; ++i, y.next()) {
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = fmaf(m[i][v], h[v], u[i][v]);
        store<E, V>(y.p(), h);
      }
    } else {
#pragma unroll
      for (int i = 0; i < K; ++i, y.next()) {
        float o[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          h[v] = here >> i & 1 ? u[i][v] : fmaf(m[i][v], h[v], u[i][v]);
          o[v] = t + i < l.len ? h[v] : 0.0f;
        }
        if (l.on && t + i < a.T) store<E, V>(y.p(), o);
      }
    }
  }
  if (!carries) return;
  if (MODE == kMaps) {
    float* to = a.ws + (int64_t)place.seg * n + column;
    to[0] = A_all;
    to[(int64_t)segments * n] = carry;
  } else if (a.h_last && k1 == chunks) {
    a.h_last[column] = carry;
  }
}

__global__ void __launch_bounds__(kThreads) k_no_steps(const float* from, float* to, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) to[i] = from ? from[i] : 0.0f;
}

// ---- backward

// A segment's map of the gradient behind it to the one in front of it: g and dy are read, 5.0 TB/s.
template <typename E, int V, int N>
__global__ void __launch_bounds__(8192 / N) k_backward_maps(RecurArgs a, int chunks, int per, int segments) {
  using S = Shape<E, V, N>;
  constexpr int K = S::K;
  __shared__ float runs[2][2][S::kRuns][kColumns];
  const int64_t n = (int64_t)a.P * a.B * a.C, first = (int64_t)blockIdx.x * kColumns, column = first + threadIdx.x;
  const int at = threadIdx.x % S::kLanes, run = threadIdx.x / S::kLanes;
  const Lane l = lane_at(a, first + at * V);
  const int k0 = blockIdx.y * per, k1 = min(k0 + per, chunks);
  float bias[V];
  bias_of<V>(a, l, bias);
  Strip<E, V, K> g, dy;
  Resets<K> starts;
  const auto fetch = [&](int k) {
    const int t = k * kRecurChunk + run * K;
    if (!__any(t < l.len)) return;
    g.load(a.g, l, t, a.T);
    dy.load(a.dy, l, t, a.T);
    starts.load(a, l, t);
  };
  fetch(k1 - 1);
  float d = 0.0f, A_all = 1.0f;
  for (int k = k1 - 1; k >= k0; --k) {
    const int t = k * kRecurChunk + run * K;
    const unsigned here = starts.bits(a, l, t);
    float A[V], D[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; D[v] = 0.0f; }
    if (__all(t + K <= l.len) && !__any(here != 0)) {
#pragma unroll
      for (int i = K - 1; i >= 0; --i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float q = gate<E>(element<V>(g.v[i], v) + bias[v]).a;
          D[v] = q * (D[v] + element<V>(dy.v[i], v));
          A[v] *= q;
        }
    } else {
#pragma unroll
      for (int i = K - 1; i >= 0; --i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float q = gate<E>(element<V>(g.v[i], v) + bias[v]).a;
          const bool live = t + i < l.len;
          const float next = here >> i & 1 ? 0.0f : q * (D[v] + element<V>(dy.v[i], v));
          D[v] = live ? next : D[v];
          A[v] = live ? A[v] * q : A[v];
        }
#pragma unroll
      for (int v = 0; v < V; ++v) A[v] = here ? -0.0f : A[v];
    }
    if (k > k0) fetch(k - 1);
    auto& sA = runs[k & 1][0];
    auto& sD = runs[k & 1][1];
#pragma unroll
    for (int v = 0; v < V; ++v) { sA[run][at * V + v] = A[v]; sD[run][at * V + v] = D[v]; }
    sync_lds();
    if (threadIdx.x < kColumns) {
#pragma unroll 8
      for (int i = S::kRuns - 1; i >= 0; --i) {
        const float Ai = sA[i][threadIdx.x];
        A_all = compose(A_all, Ai);
        d = apply(Ai, sD[i][threadIdx.x], d);
      }
    }
  }
  if (threadIdx.x < kColumns && column < n) {
    if (a.dh_last && (int)blockIdx.y == segments - 1) first_of(a, n, segments)[column] = a.dh_last[column];
    float* to = a.ws + (int64_t)blockIdx.y * n + column;
    to[0] = A_all;
    to[(int64_t)segments * n] = d;
  }
}

// dx and dg, and the sums of dg over the segment to `sums` [segments, columns].  States are found again from those in front
// of the tiles, at an LDS walk's cost; gates too: kept ones would be another array to write and read.  Bound by memory, 5
// elements a step and column: 80 agents of 8 x 512 x 256 in bf16 199 us, 4.2 TB/s; 2 of 2 x 16383 x 512 in fp16 75 us, 4.5,
// behind 27 for the maps.  The chain (23 agents of 3 x 777 x 129, fp32, single elements, ragged: 36 us) also waits for its
// hand-overs.
template <typename E, int V, int N, int MODE>
__global__ void __launch_bounds__(8192 / N, 2) k_backward(RecurArgs a, int chunks, int per, int segments, float* sums) {
  using S = Shape<E, V, N>;
  constexpr int K = S::K;
  __shared__ float runs[2][3][S::kRuns][kColumns];             // [tile parity][A; H, then states in front; D, then gradients behind]
  __shared__ float quarter[4][2][kColumns];
  const int64_t n = (int64_t)a.P * a.B * a.C;
  const Place place = place_of<MODE>(a, n, segments, true);
  const int at = threadIdx.x % S::kLanes, run = threadIdx.x / S::kLanes, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Lane l = lane_at(a, place.first + at * V);
  const int k0 = place.seg * per, k1 = MODE == kChain ? k0 + 1 : min(k0 + per, chunks);
  float bias[V];
  bias_of<V>(a, l, bias);
  Strip<E, V, K> x, g, dy;
  Resets<K> starts;
  const auto fetch = [&](int k) {
    const int t = k * kRecurChunk + run * K;
    if (!__any(t < l.len)) return;
    g.load(a.g, l, t, a.T);
    x.load(a.x, l, t, a.T);
    dy.load(a.dy, l, t, a.T);
    starts.load(a, l, t);
  };
  fetch(k1 - 1);
  // a column per lane: wavefront 0 carries the gradient from tile to tile, wavefront 1 takes states from `states`
  const int64_t column = place.first + lane, row = column / a.C;
  const bool valid = column < n;
  float d = 0.0f;
  if (a.dh_last && valid && (MODE != kChain || k1 == chunks)) d = MODE == kSegments ? first_of(a, n, segments)[column] : a.dh_last[column];
  if (MODE == kSegments) d = enter(a, n, column, segments, segments - 1, segments - 1 - place.seg, -1, d, quarter);
  const float* states = a.states + row * chunks * a.C + (column - row * a.C);
  const int64_t dx_at = base(a.dx, l) + l.c, dg_at = base(a.dg, l) + l.c;
  float sum[V];
#pragma unroll
  for (int v = 0; v < V; ++v) sum[v] = 0.0f;

  for (int k = k1 - 1; k >= k0; --k) {
    const int t = k * kRecurChunk + run * K;
    const unsigned here = starts.bits(a, l, t);
    const bool full = __all(t + K <= l.len), plain = full && !__any(here != 0);
    const float state = wave == 1 && valid ? states[(int64_t)k * a.C] : 0.0f;
    // gates, inputs (then: state in front minus input) and gradients of the steps
    float A[V], H[V], D[V], ga[K][V], gb[K][V], w[K][V], ds[K][V];
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = D[v] = 0.0f; }
    if (plain) {
#pragma unroll
      for (int i = 0; i < K; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const Gate q = gate<E>(element<V>(g.v[i], v) + bias[v]);
          ga[i][v] = q.a;
          gb[i][v] = q.b;
          w[i][v] = element<V>(x.v[i], v);
          ds[i][v] = element<V>(dy.v[i], v);
          H[v] = fmaf(q.a, H[v], q.b * w[i][v]);
          A[v] *= q.a;
        }
#pragma unroll
      for (int i = K - 1; i >= 0; --i)
#pragma unroll
        for (int v = 0; v < V; ++v) D[v] = ga[i][v] * (D[v] + ds[i][v]);
    } else {
#pragma unroll
      for (int i = 0; i < K; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const Gate q = gate<E>(element<V>(g.v[i], v) + bias[v]);
          const bool live = t + i < l.len;
          ga[i][v] = live ? q.a : 1.0f;
          gb[i][v] = live ? q.b : 0.0f;
          w[i][v] = live ? element<V>(x.v[i], v) : 0.0f;
          ds[i][v] = live ? element<V>(dy.v[i], v) : 0.0f;
          const float u = gb[i][v] * w[i][v];
          H[v] = here >> i & 1 ? u : fmaf(ga[i][v], H[v], u);
          A[v] *= ga[i][v];
        }
#pragma unroll
      for (int i = K - 1; i >= 0; --i)
#pragma unroll
        for (int v = 0; v < V; ++v) D[v] = here >> i & 1 ? 0.0f : ga[i][v] * (D[v] + ds[i][v]);
#pragma unroll
      for (int v = 0; v < V; ++v) A[v] = here ? -0.0f : A[v];
    }
    if (MODE != kChain && k > k0) fetch(k - 1);
    auto& sA = runs[k & 1][0];
    auto& sH = runs[k & 1][1];
    auto& sD = runs[k & 1][2];
#pragma unroll
    for (int v = 0; v < V; ++v) { sA[run][at * V + v] = A[v]; sH[run][at * V + v] = H[v]; sD[run][at * V + v] = D[v]; }
    sync_lds();
    if (wave == 0) {
      if (MODE == kChain && k1 < chunks && valid) d = taken_over(words_of(a) + (int64_t)(place.seg + 1) * n + column);
#pragma unroll 8
      for (int i = S::kRuns - 1; i >= 0; --i) {
        const float Ai = sA[i][lane], Di = sD[i][lane];
        sD[i][lane] = d;
        d = apply(Ai, Di, d);
      }
      if (MODE == kChain && place.seg > 0 && valid) hand_over(words_of(a) + (int64_t)place.seg * n + column, d);
    } else if (wave == 1) {
      float s = state;
#pragma unroll 8
      for (int i = 0; i < S::kRuns; ++i) {
        const float Ai = sA[i][lane], Hi = sH[i][lane];
        sH[i][lane] = s;
        s = apply(Ai, Hi, s);
      }
    }
    sync_lds();
    float h[V], e[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { h[v] = sH[run][at * V + v]; e[v] = sD[run][at * V + v]; }
    Walk<E, V> px(a.dx, dx_at, t + K - 1), pg(a.dg, dg_at, t + K - 1);
    px.step = -px.step;
    pg.step = -pg.step;
    if (plain) {
#pragma unroll
      for (int i = 0; i < K; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float u = gb[i][v] * w[i][v];
          w[i][v] = h[v] - w[i][v];
          h[v] = fmaf(ga[i][v], h[v], u);
        }
#pragma unroll
      for (int i = K - 1; i >= 0; --i, px.next(), pg.next()) {
        float dx[V], dg[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float all = e[v] + ds[i][v];
          dx[v] = all * gb[i][v];
          e[v] = ga[i][v] * all;
          dg[v] = dx[v] * w[i][v] * ga[i][v];
          sum[v] += dg[v];
        }
        store<E, V>(px.p(), dx);
        store<E, V>(pg.p(), dg);
      }
    } else {
#pragma unroll
      for (int i = 0; i < K; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const bool r = here >> i & 1;
          const float u = gb[i][v] * w[i][v];
          w[i][v] = (r ? 0.0f : h[v]) - w[i][v];
          h[v] = r ? u : fmaf(ga[i][v], h[v], u);
        }
#pragma unroll
      for (int i = K - 1; i >= 0; --i, px.next(), pg.next()) {
        float dx[V], dg[V];
        const bool live = t + i < l.len;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float all = e[v] + ds[i][v];
          dx[v] = live ? all * gb[i][v] : 0.0f;
          dg[v] = live ? dx[v] * w[i][v] * ga[i][v] : 0.0f;
          e[v] = here >> i & 1 ? 0.0f : ga[i][v] * all;
          sum[v] += dg[v];
        }
        if (l.on && t + i < a.T) {
          store<E, V>(px.p(), dx);
          store<E, V>(pg.p(), dg);
        }
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
#pragma unroll 8
    for (int i = 0; i < S::kRuns; ++i) s += part[i][lane];
    sums[(int64_t)place.seg * n + column] = s;
  }
}

// dbias from the sums of every segment and sequence: a workgroup per 64 of the P * C results, a quarter of the terms per
// wavefront.
__global__ void __launch_bounds__(kThreads) k_bias_sum(const float* sums, float* dbias, int P, int B, int C, int segments) {
  __shared__ float part[4][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 64 + lane, n = (int64_t)P * B * C;
  const int terms = segments * B, q = (terms + 3) / 4, lo = min(wave * q, terms), hi = min(lo + q, terms);
  const bool on = i < (int64_t)P * C;
  const float* from = sums + (on ? i / C * B * C + i % C : 0);
  float v = 0.0f;
#pragma unroll 8
  for (int k = lo; k < hi; ++k) v += from[(int64_t)(k / B) * n + (int64_t)(k % B) * C];
  part[wave][lane] = v;
  __syncthreads();
  if (wave == 0 && on) dbias[i] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
}

// ---- single steps

// V channels of a row per lane; memory's latency for few rows (10 of 256 channels: 2.8 us), its rate for many (80 agents of
// 256 rows x 256 in bf16: 11.8 us, 73 MB at 6.2 TB/s, which the Infinity Cache gives and HBM would not).
template <typename E, int V>
__global__ void __launch_bounds__(kThreads) k_step(RecurArgs a) {
  typedef typename Vec<E, V>::type vec;
  typedef typename Vec<float, V>::type fvec;
  const Lane l = lane_at(a, ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * V);
  if (!l.on) return;
  const int slot = a.slots ? a.slots[l.row] : l.b;
  float h[V] = {};
  if (slot >= 0 && slot < a.n_slots) {
    fvec* state = (fvec*)(a.state + ((int64_t)l.p * a.n_slots + slot) * a.C + l.c);
    const vec g = *(const vec*)((const E*)a.g.data + base(a.g, l) + l.c), x = *(const vec*)((const E*)a.x.data + base(a.x, l) + l.c);
    const bool r = a.reset.data && ((const uint8_t*)a.reset.data)[base(a.reset, l)] != 0;
    const fvec before = *state;
    fvec bias = {}, after;
    if (a.bias) bias = *(const fvec*)(a.bias + (int64_t)l.p * a.C + l.c);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Gate q = gate<E>(element<V>(g, v) + element<V>(bias, v));
      const float u = q.b * element<V>(x, v);
      h[v] = r ? u : fmaf(q.a, element<V>(before, v), u);
      if constexpr (V == 1) after = h[v]; else after[v] = h[v];
    }
    *state = after;
  }
  store<E, V>((typename Walk<E, V>::pointer)((E*)a.y.data + base(a.y, l) + l.c), h);
}

// ---- launches

unsigned blocks(int64_t n) { return (unsigned)((n + kThreads - 1) / kThreads); }

// Elements of a tile per lane: workgroups of 256 threads for 32, of 512 for 16.  The forward kernels of long sequences are
// ahead with 32 (one sequence of 65536 x 256 41.1 us, with 16 43.0; with its backward pass, 80 agents of 8 x 512 x 256 321 /
// 328), chains, whose tiles wait for each other, with 16 (10 agents of 4 x 1000 x 256 31.3 / 34.2); the backward kernel holds
// twice as much per element, with 32 it spills (80 agents: 552), and with 8 gains nothing (333).
constexpr int kElements = 32, kElementsChain = 16, kElementsBack = 16;

// How sequences are shared, by groups of 64 columns and tiles of 128 steps; us of a forward and a backward pass.
// kWhole from 256 groups on, where the columns alone fill the chip: 256 groups of 4 tiles in bf16 39, as chains 55; 512 of 16
// 222 / 308; 2560 of 4 290 / 383; fp32 256 of 4 53 / 65.  But in fp32, where such calls are bound by memory alone, chains,
// whose workgroups are many and short, leave no CU idle at the end: 320 groups of 16 tiles 263, whole 321; 640 of 8 261 / 286;
// 2560 of 8 982 / 1047 (512 of 8: 224 / 220; 256 of 8: 117 / 104).
// A chain takes 1.25 us a tile from one workgroup to the next, segments read two thirds more: with few columns segments
// are ahead, from 64 groups in fp32 (128 of 16 bits) on chains.  fp32, 32 groups of 16 tiles: chains 67, segments 47; of
// 32: 106 / 92; 64 of 16: 75 / 90; of 128: 463 / 631; bf16, 64 of 16: 66 / 61; of 128: 376 / 337; 128 of 16: 88 / 96; of 128:
// 595 / 661.
struct Cut { int mode, chunks, per, segments; };
constexpr int kMaxSegments = 128, kWholeFrom = 256, kChainBytesFrom = 256, kWholeTiles = 8;
constexpr int64_t kChainTilesMost = 1 << 22; // workgroups of 512 work items, below 2^32 in all
Cut cut_of(int64_t P, int64_t B, int64_t T, int64_t C, int64_t element) {
  const int64_t groups = (P * B * C + kColumns - 1) / kColumns, chunks = recur_chunks(T);
  const bool chains = groups * chunks <= kChainTilesMost;
  if (chunks <= 1 || (groups >= kWholeFrom && (element == 2 || chunks < kWholeTiles || !chains))) return {kWhole, (int)chunks, (int)chunks, 1};
  if (chains && groups * element >= kChainBytesFrom) return {kChain, (int)chunks, 1, (int)chunks};
  int64_t want = (1024 + groups - 1) / groups;
  if (want > kMaxSegments) want = kMaxSegments;
  if (want > chunks) want = chunks;
  const int64_t per = (chunks + want - 1) / want;
  return {kSegments, (int)chunks, (int)per, (int)((chunks + per - 1) / per)};
}

// Whether every row of an array can be read in vectors of 4 elements.
bool wide(const pop_sequence& s, int64_t bytes) {
  return (uintptr_t)s.data % (4 * bytes) == 0 && s.agent % 4 == 0 && s.row % 4 == 0 && s.step % 4 == 0;
}

dim3 grid_of(const Cut& c, int64_t n) {
  const unsigned groups = (unsigned)((n + kColumns - 1) / kColumns);
  return c.mode == kChain ? dim3(groups * c.segments) : dim3(groups, c.segments);
}
void clear(const RecurArgs& a, const Cut& c, int64_t n, hipStream_t s) {
  const int64_t words = n * c.segments + 1;
  k_clear<<<blocks(words), kThreads, 0, s>>>((unsigned long long*)a.ws, words);
}

template <typename E, int V> void forward(const RecurArgs& a, const Cut& c, int64_t n, hipStream_t s) {
  const dim3 grid = grid_of(c, n);
  if (c.mode == kWhole) {
    k_forward<E, V, kElements, kWhole><<<grid, 8192 / kElements, 0, s>>>(a, c.chunks, c.per, c.segments);
  } else if (c.mode == kChain) {
    clear(a, c, n, s);
    k_forward<E, V, kElementsChain, kChain><<<grid, 8192 / kElementsChain, 0, s>>>(a, c.chunks, c.per, c.segments);
  } else {
    k_forward<E, V, kElements, kMaps><<<grid, 8192 / kElements, 0, s>>>(a, c.chunks, c.per, c.segments);
    k_forward<E, V, kElements, kSegments><<<grid, 8192 / kElements, 0, s>>>(a, c.chunks, c.per, c.segments);
  }
}
template <typename E> hipError_t forward(const RecurArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.P * a.B * a.C;
  if (a.T == 0) {
    if (a.h_last) k_no_steps<<<blocks(n), kThreads, 0, s>>>(a.h0, a.h_last, n);
    return hipGetLastError();
  }
  const int64_t e = sizeof(E);
  const Cut c = cut_of(a.P, a.B, a.T, a.C, e);
  if (a.C % 4 == 0 && wide(a.x, e) && wide(a.g, e) && wide(a.y, e)) forward<E, 4>(a, c, n, s);
  else forward<E, 1>(a, c, n, s);
  return hipGetLastError();
}

template <typename E, int V> void backward(const RecurArgs& a, const Cut& c, int64_t n, float* sums, hipStream_t s) {
  const dim3 grid = grid_of(c, n);
  if (c.mode == kWhole) {
    k_backward<E, V, kElementsBack, kWhole><<<grid, 8192 / kElementsBack, 0, s>>>(a, c.chunks, c.per, c.segments, sums);
  } else if (c.mode == kChain) {
    clear(a, c, n, s);
    k_backward<E, V, kElementsBack, kChain><<<grid, 8192 / kElementsBack, 0, s>>>(a, c.chunks, c.per, c.segments, sums);
  } else {
    k_backward_maps<E, V, kElements><<<grid, 8192 / kElements, 0, s>>>(a, c.chunks, c.per, c.segments);
    k_backward<E, V, kElementsBack, kSegments><<<grid, 8192 / kElementsBack, 0, s>>>(a, c.chunks, c.per, c.segments, sums);
  }
}
template <typename E> hipError_t backward(const RecurArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.P * a.B * a.C, nb = (int64_t)a.P * a.C;
  if (a.T == 0) {
    if (a.dh0) k_no_steps<<<blocks(n), kThreads, 0, s>>>(a.dh_last, a.dh0, n);
    if (a.dbias) k_no_steps<<<blocks(nb), kThreads, 0, s>>>(nullptr, a.dbias, nb);
    return hipGetLastError();
  }
  const int64_t e = sizeof(E);
  const Cut c = cut_of(a.P, a.B, a.T, a.C, e);
  float* sums = a.ws + 2 * (n * c.segments + 1);
  if (a.C % 4 == 0 && wide(a.x, e) && wide(a.g, e) && wide(a.dy, e) && wide(a.dx, e) && wide(a.dg, e)) backward<E, 4>(a, c, n, sums, s);
  else backward<E, 1>(a, c, n, sums, s);
  if (a.dbias) k_bias_sum<<<(unsigned)((nb + 63) / 64), kThreads, 0, s>>>(sums, a.dbias, a.P, a.B, a.C, c.segments);
  return hipGetLastError();
}

template <typename E> hipError_t step(const RecurArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.P * a.B * a.C, e = sizeof(E);
  const auto row = [&](const pop_sequence& q) { return (uintptr_t)q.data % (4 * e) == 0 && q.agent % 4 == 0 && q.row % 4 == 0; };
  if (a.C % 4 == 0 && row(a.x) && row(a.g) && row(a.y) && (uintptr_t)a.state % 16 == 0 && (uintptr_t)a.bias % 16 == 0)
    k_step<E, 4><<<blocks(n / 4), kThreads, 0, s>>>(a);
  else
    k_step<E, 1><<<blocks(n), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace recur
}  // namespace

int64_t recur_workspace_floats(int64_t P, int64_t B, int64_t T, int64_t C, int64_t element) {
  if (T == 0) return 0;
  const recur::Cut c = recur::cut_of(P, B, T, C, element);
  return P * B * C * (3 * c.segments + (c.mode == recur::kSegments)) + 2;      // maps or words (and the ticket), sums, first states
}

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
