// Newton-Schulz orthogonalisation of stacks of matrices, and the Muon step around it (operators.h).
//
//   X = U / (|U| + eps);  steps times:  A = X X^T,  B = k1 A + k2 A A,  X = k0 X + B X
//
// with X of m x n, m <= n (matrices with more rows than columns are taken transposed).  All matrices of a call advance
// together: per step one launch for A, one for B, one for X; A and B are symmetric, so only their tiles on and above
// the diagonal are computed.
//
// Products on v_mfma_f32_32x32x16_f16 from operands in two fp16 halves, x = hi + lo with 11 bits each, held in units
// (powers of two, Units below) that keep the largest possible entry just below 2^15, so that lo keeps its bits for
// entries down to 2^-14 of the largest: x y = hi hi + hi lo + lo hi, what is left out is below 2^-22 |x y|.  Three instructions in
// place of sixteen of the fp32 ones.
//
// Operands lie in the workspace as the instruction takes them: blocks of 32 rows x 16 contraction indices, 64 lanes
// of 8 halves (lane l: row l & 31, indices 8 (l >> 5) ..), the hi block in front of the lo block, 2 KB together,
// blocks of one row band adjacent.  Both operands have the contraction index inside, so X is kept in both orders.
#include <hip/hip_runtime.h>
#include "operators.h"

namespace pop {
namespace {
namespace ns {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kPair = 1024;                 // halves of a hi and a lo block

// Where the arrays of one matrix lie, in halves from the start of its workspace.
struct Place {
  int mb, nb;                               // 32-row bands of m and n
  int64_t x, xt[2], a, b, size;             // X [m rows, n inside], X^T [n rows, m inside] twice, A, B
};
__host__ __device__ inline Place place(int rows, int cols) {
  Place p;
  p.mb = ((rows < cols ? rows : cols) + 31) / 32;
  p.nb = ((rows < cols ? cols : rows) + 31) / 32;
  const int64_t xs = (int64_t)p.mb * p.nb * 2 * kPair, as = (int64_t)p.mb * p.mb * 2 * kPair;
  p.x = 0; p.xt[0] = xs; p.xt[1] = 2 * xs; p.a = 3 * xs; p.b = 3 * xs + as;
  p.size = 3 * xs + 2 * as;
  return p;
}
constexpr int kSumParts = 256;              // most partial sums of one matrix's squares
constexpr int kSums = kSumParts + 1;        // behind them |X| of the first X
__host__ __device__ inline int64_t part_elements(int rows, int cols) {
  const int64_t n = (int64_t)rows * cols, a = (n + kSumParts - 1) / kSumParts;
  return a > 8192 ? a : 8192;
}
__host__ __device__ inline int parts(int rows, int cols) {
  const int64_t e = part_elements(rows, cols);
  return (int)(((int64_t)rows * cols + e - 1) / e);
}

__host__ __device__ inline int64_t sum_bytes(int count) { return ((int64_t)count * kSums * 8 + 255) / 256 * 256; }

// Units of X, A = X X^T and B = k1 A + k2 A A in front of a step: powers of two by which entries are held multiplied.
// No entry exceeds the largest singular value, which is below `most` whatever the matrix, and below gain[step] |X| of
// the first X where eps made that small.  (The limits on the exponents keep the units and what they divide finite:
// an X below 2^-100 is as good as none, and an A or B below 2^-60 makes no difference to X.)
struct Units { float x, a, b; };
__device__ inline float unit_of(float most, int limit) { return ldexpf(1.0f, min(14 - ilogbf(fmaxf(most, 0x1p-120f)), limit)); }
__device__ inline Units units_of(const NsCall& c, int step, float start) {
  const float x = fminf(c.most, start * c.gain[step]), a = x * x;
  return {unit_of(x, 100), unit_of(a, 60), unit_of(fabsf(c.coef[step][1]) * a + fabsf(c.coef[step][2]) * a * a, 60)};
}

struct Work {                               // a launch: workgroups of every layer
  int first[POP_MUON_MAX_LAYERS + 1];       // first workgroup of a layer
  int per[POP_MUON_MAX_LAYERS];             // workgroups of one matrix
  int64_t ws[POP_MUON_MAX_LAYERS];          // bytes to the layer's workspace
};

struct At { int layer, matrix, unit; };
__device__ inline At find(const Work& w) {
  int k = 0;
  while ((int)blockIdx.x >= w.first[k + 1]) ++k;
  const int i = (int)blockIdx.x - w.first[k];
  return {k, i / w.per[k], i % w.per[k]};
}

// a layer's workspace: sums [count, kSums], then the matrices
__device__ inline double* sums_of(char* ws, const Work& w, const At& at) { return (double*)(ws + w.ws[at.layer]) + (int64_t)at.matrix * kSums; }
__device__ inline _Float16* halves_of(char* ws, const Work& w, const At& at, const NsLayer& l, const Place& p) {
  return (_Float16*)(ws + w.ws[at.layer] + sum_bytes(l.count)) + (int64_t)at.matrix * p.size;
}

// ---- momentum and norms

constexpr int kThreads = 256;

template <typename G>
__global__ void __launch_bounds__(kThreads) k_norms(NsCall c, Work w, char* ws) {
  __shared__ double red[kThreads];
  const At at = find(w);
  const NsLayer& l = c.layer[at.layer];
  const int64_t e = part_elements(l.rows, l.cols), n = (int64_t)l.rows * l.cols;
  const int64_t lo = at.unit * e, hi = lo + e < n ? lo + e : n;
  const float mu = c.hparams ? c.hparams[3 * at.matrix + 1] : 0.0f;
  double sum = 0.0;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const int r = (int)(i / l.cols), k = (int)(i % l.cols);
    float u = (float)((const G*)l.g)[at.matrix * l.g_matrix + r * l.g_row + k];
    if (c.hparams) {
      float* m = l.momentum + at.matrix * l.m_matrix + r * l.m_row + k;
      const float v = fmaf(mu, *m, u);
      *m = v;
      u = c.nesterov ? fmaf(mu, v, u) : v;
    }
    sum += (double)u * u;
  }
  red[threadIdx.x] = sum;
  __syncthreads();
  for (int s = kThreads / 2; s > 0; s /= 2) {
    if ((int)threadIdx.x < s) red[threadIdx.x] += red[threadIdx.x + s];
    __syncthreads();
  }
  if (threadIdx.x == 0) sums_of(ws, w, at)[at.unit] = red[0];
}

// |U| from the partial sums, the same in every workgroup
__device__ inline double norm_of(const double* sums, int n, double* red) {
  red[threadIdx.x] = (int)threadIdx.x < n ? sums[threadIdx.x] : 0.0;
  __syncthreads();
  for (int s = kThreads / 2; s > 0; s /= 2) {
    if ((int)threadIdx.x < s) red[threadIdx.x] += red[threadIdx.x + s];
    __syncthreads();
  }
  return sqrt(red[0]);
}

// ---- blocks of operands

// Accumulator tile of 32 x 32: register 4 q + r of lane l is element (row i = 8 q + 4 (l >> 5) + r, column j = l & 31).
// `put_turned` writes it with j as the row and i inside (four i are adjacent); `put` with i as the row and j inside, by
// way of 32 x 33 words of LDS of this wavefront.  band: 32-row band of the target, inside: its 32 inner indices' number.
struct Halves { _Float16 hi, lo; };
__device__ inline Halves split(float v) {
  const _Float16 hi = (_Float16)v;
  return {hi, (_Float16)(v - (float)hi)};
}
__device__ inline int64_t pair_at(int band, int inside16, int bands_inside) { return ((int64_t)band * bands_inside * 2 + inside16) * kPair; }

__device__ inline void put_turned(_Float16* base, int band, int inside, int bands_inside, const f32x16& v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f16x4 hi, lo;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const Halves h = split(v[4 * q + r]);
      hi[r] = h.hi;
      lo[r] = h.lo;
    }
    _Float16* to = base + pair_at(band, 2 * inside + (q >> 1), bands_inside) + ((lane & 31) + 32 * (q & 1)) * 8 + 4 * (lane >> 5);
    *(f16x4*)to = hi;
    *(f16x4*)(to + kPair / 2) = lo;
  }
}
__device__ inline void put(_Float16* base, int band, int inside, int bands_inside, const f32x16& v, float* scratch) {
  const int lane = threadIdx.x & 63;
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < 16; ++i) scratch[(8 * (i >> 2) + 4 * (lane >> 5) + (i & 3)) * 33 + (lane & 31)] = v[i];
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    f16x8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Halves h = split(scratch[(lane & 31) * 33 + 16 * s + 8 * (lane >> 5) + i]);
      hi[i] = h.hi;
      lo[i] = h.lo;
    }
    _Float16* to = base + pair_at(band, 2 * inside + s, bands_inside) + lane * 8;
    *(f16x8*)to = hi;
    *(f16x8*)(to + kPair / 2) = lo;
  }
  __builtin_amdgcn_wave_barrier();
}
// what put_turned wrote
__device__ inline f32x16 get_turned(const _Float16* base, int band, int inside, int bands_inside) {
  const int lane = threadIdx.x & 63;
  f32x16 v;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const _Float16* from = base + pair_at(band, 2 * inside + (q >> 1), bands_inside) + ((lane & 31) + 32 * (q & 1)) * 8 + 4 * (lane >> 5);
    const f16x4 hi = *(const f16x4*)from, lo = *(const f16x4*)(from + kPair / 2);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[4 * q + r] = (float)hi[r] + (float)lo[r];
  }
  return v;
}

// ---- X in both orders

template <typename G>
__global__ void __launch_bounds__(kThreads) k_start(NsCall c, Work w, char* ws) {
  __shared__ double red[kThreads];
  __shared__ float scratch[4][32 * 33];
  const At at = find(w);
  const NsLayer& l = c.layer[at.layer];
  const Place p = place(l.rows, l.cols);
  double* sums = sums_of(ws, w, at);
  const double norm = norm_of(sums, parts(l.rows, l.cols), red), inv = 1.0 / (norm + (double)c.eps);
  const float start = (float)(norm * inv);
  if (at.unit == 0 && threadIdx.x == 0) sums[kSumParts] = start;
  const double scale = inv * units_of(c, 0, start).x;
  const float mu = c.hparams ? c.hparams[3 * at.matrix + 1] : 0.0f;
  const bool turned = l.rows > l.cols;
  const int cb = turned ? p.mb : p.nb, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int block = at.unit * 4 + wave;
  if (block >= p.mb * p.nb) return;
  const int ib = block / cb, jb = block % cb;
  f32x16 v;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int r = ib * 32 + 8 * (k >> 2) + 4 * (lane >> 5) + (k & 3), j = jb * 32 + (lane & 31);
    float u = 0.0f;
    if (r < l.rows && j < l.cols) {
      const bool plain = !c.hparams || c.nesterov;
      const float g = plain ? (float)((const G*)l.g)[at.matrix * l.g_matrix + r * l.g_row + j] : 0.0f;
      const float m = c.hparams ? l.momentum[at.matrix * l.m_matrix + r * l.m_row + j] : 0.0f;
      u = (float)((double)(c.hparams ? (c.nesterov ? fmaf(mu, m, g) : m) : g) * scale);
    }
    v[k] = u;
  }
  _Float16* base = halves_of(ws, w, at, l, p);
  // rows of the matrix are m unless it is turned
  put_turned(base + (turned ? p.x : p.xt[0]), jb, ib, turned ? p.nb : p.mb, v);
  put(base + (turned ? p.xt[0] : p.x), ib, jb, turned ? p.mb : p.nb, v, scratch[wave]);
}

// ---- products

enum { kGram = 0, kPoly = 1, kApply = 2, kLast = 3 };
constexpr int kTile = 4;                    // 32-row bands of a workgroup's tile: 2 x 2 wavefronts of 2 x 2 blocks

__device__ inline f32x16 mfma(const f16x8& a, const f16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

template <int MODE, typename G>
__global__ void __launch_bounds__(kThreads) k_product(NsCall c, Work w, char* ws, int step) {
  __shared__ float scratch[4][32 * 33];
  const At at = find(w);
  const NsLayer& l = c.layer[at.layer];
  const Place p = place(l.rows, l.cols);
  const bool turned = MODE == kLast && l.rows > l.cols;
  _Float16* base = halves_of(ws, w, at, l, p);
  const _Float16 *xt = base + p.xt[step & 1];
  // left operand: rows i, right operand: rows j, `inner` blocks of 16
  const _Float16* left = MODE == kGram ? base + p.x : MODE == kPoly ? base + p.a : turned ? xt : base + p.b;
  const _Float16* right = MODE == kGram ? base + p.x : MODE == kPoly ? base + p.a : turned ? base + p.b : xt;
  const int ibands = turned ? p.nb : p.mb, jbands = MODE < kApply || turned ? p.mb : p.nb;
  const int inner = 2 * (MODE == kGram ? p.nb : p.mb);
  int ti, tj;
  if (MODE < kApply) {                      // tiles on and above the diagonal
    const int t = (p.mb + kTile - 1) / kTile;
    ti = 0;
    int u = at.unit;
    while (u >= t - ti) { u -= t - ti; ++ti; }
    tj = ti + u;
  } else {
    const int t = (jbands + kTile - 1) / kTile;
    ti = at.unit / t;
    tj = at.unit % t;
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int i0 = ti * kTile + (wave >> 1) * 2, j0 = tj * kTile + (wave & 1) * 2;
  if (i0 >= ibands || j0 >= jbands) return;
  const _Float16 *lp[2], *rp[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {             // a band beyond the edge: the last one again, not stored
    lp[s] = left + (int64_t)min(i0 + s, ibands - 1) * inner * kPair + lane * 8;
    rp[s] = right + (int64_t)min(j0 + s, jbands - 1) * inner * kPair + lane * 8;
  }
  f32x16 acc[2][2] = {};
  for (int k = 0; k < inner; ++k) {
    f16x8 lh[2], ll[2], rh[2], rl[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      lh[s] = *(const f16x8*)(lp[s] + (int64_t)k * kPair);
      ll[s] = *(const f16x8*)(lp[s] + (int64_t)k * kPair + kPair / 2);
      rh[s] = *(const f16x8*)(rp[s] + (int64_t)k * kPair);
      rl[s] = *(const f16x8*)(rp[s] + (int64_t)k * kPair + kPair / 2);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        acc[i][j] = mfma(lh[i], rl[j], acc[i][j]);
        acc[i][j] = mfma(ll[i], rh[j], acc[i][j]);
        acc[i][j] = mfma(lh[i], rh[j], acc[i][j]);
      }
  }
  const float start = (float)sums_of(ws, w, at)[kSumParts];
  const Units u = units_of(c, step, start);
  const float next = MODE == kLast ? 1.0f : units_of(c, step + 1, start).x;
  const float k0 = c.coef[step][0], k1 = c.coef[step][1], k2 = c.coef[step][2];
#pragma unroll
  for (int bi = 0; bi < 2; ++bi)
#pragma unroll
    for (int bj = 0; bj < 2; ++bj) {
      const int ib = i0 + bi, jb = j0 + bj;
      if (ib >= ibands || jb >= jbands) continue;
      f32x16 v = acc[bi][bj];
      if (MODE == kGram) {
        v = v * (1.0f / u.x) * (u.a / u.x);
      } else if (MODE == kPoly) {
        const f32x16 a = get_turned(base + p.a, jb, ib, p.mb);
        v = v * (1.0f / u.a) * (k2 * (u.b / u.a)) + a * (k1 * (u.b / u.a));
      } else {
        const f32x16 x = turned ? get_turned(base + p.x, jb, ib, p.nb) : get_turned(xt, jb, ib, p.mb);
        v = v * (1.0f / u.b) * (next / u.x) + x * (k0 * (next / u.x));
      }
      if (MODE == kGram || MODE == kPoly) {
        _Float16* to = base + (MODE == kGram ? p.a : p.b);
        put_turned(to, jb, ib, p.mb, v);
        if (ti != tj) put(to, ib, jb, p.mb, v, scratch[wave]);
      } else if (MODE == kApply) {
        put_turned(base + p.xt[~step & 1], jb, ib, p.mb, v);
        put(base + p.x, ib, jb, p.nb, v, scratch[wave]);
      } else {
        const int j = jb * 32 + (lane & 31);
        const float lr = c.hparams ? c.hparams[3 * at.matrix] : 0.0f, wd = c.hparams ? c.hparams[3 * at.matrix + 2] : 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int r = ib * 32 + 8 * (k >> 2) + 4 * (lane >> 5) + (k & 3);
          if (r >= l.rows || j >= l.cols) continue;
          if (c.hparams) {
            float* to = l.weight + at.matrix * l.w_matrix + r * l.w_row + j;
            *to = fmaf(-lr * l.scale, v[k], *to * fmaf(-lr, wd, 1.0f));
          } else {
            ((G*)l.out)[at.matrix * l.out_matrix + r * l.out_row + j] = (G)v[k];
          }
        }
      }
    }
}

// no steps: X itself
template <typename G>
__global__ void __launch_bounds__(kThreads) k_no_steps(NsCall c, Work w, char* ws) {
  __shared__ double red[kThreads];
  const At at = find(w);
  const NsLayer& l = c.layer[at.layer];
  const float inv = (float)(1.0 / (norm_of(sums_of(ws, w, at), parts(l.rows, l.cols), red) + (double)c.eps));
  const int64_t e = part_elements(l.rows, l.cols), n = (int64_t)l.rows * l.cols;
  const int64_t lo = at.unit * e, hi = lo + e < n ? lo + e : n;
  const float* hp = c.hparams ? c.hparams + 3 * at.matrix : nullptr;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const int r = (int)(i / l.cols), k = (int)(i % l.cols);
    const float g = (float)((const G*)l.g)[at.matrix * l.g_matrix + r * l.g_row + k];
    if (hp) {
      const float m = l.momentum[at.matrix * l.m_matrix + r * l.m_row + k], u = c.nesterov ? fmaf(hp[1], m, g) : m;
      float* to = l.weight + at.matrix * l.w_matrix + r * l.w_row + k;
      *to = fmaf(-hp[0] * l.scale, u * inv, *to * fmaf(-hp[0], hp[2], 1.0f));
    } else {
      ((G*)l.out)[at.matrix * l.out_matrix + r * l.out_row + k] = (G)(g * inv);
    }
  }
}

template <typename F> bool work_of(const NsCall& c, F per, Work& w, int64_t& blocks) {
  int64_t off = 0;
  blocks = 0;
  for (int k = 0; k < c.n_layers; ++k) {
    const NsLayer& l = c.layer[k];
    w.first[k] = (int)blocks;
    w.per[k] = per(l);
    w.ws[k] = off;
    blocks += (int64_t)l.count * w.per[k];
    if (blocks >= (1ll << 24)) return false;      // 2^32 work items
    off += ns_workspace_bytes(l.count, l.rows, l.cols);
  }
  for (int k = c.n_layers; k <= POP_MUON_MAX_LAYERS; ++k) w.first[k] = (int)blocks;
  return true;
}

template <typename G> hipError_t run(const NsCall& c, char* ws, hipStream_t s) {
  const auto up = [](int v) { return (v + kTile - 1) / kTile; };
  Work sums, start, square, full;
  int64_t n_sums, n_start, n_square, n_full;
  if (!work_of(c, [](const NsLayer& l) { return parts(l.rows, l.cols); }, sums, n_sums) ||
      !work_of(c, [](const NsLayer& l) { const Place p = place(l.rows, l.cols); return (p.mb * p.nb + 3) / 4; }, start, n_start) ||
      !work_of(c, [&](const NsLayer& l) { const int t = up(place(l.rows, l.cols).mb); return t * (t + 1) / 2; }, square, n_square) ||
      !work_of(c, [&](const NsLayer& l) { const Place p = place(l.rows, l.cols); return up(p.mb) * up(p.nb); }, full, n_full))
    return hipErrorInvalidConfiguration;
  k_norms<G><<<dim3(n_sums), kThreads, 0, s>>>(c, sums, ws);
  if (c.steps == 0) {
    k_no_steps<G><<<dim3(n_sums), kThreads, 0, s>>>(c, sums, ws);
    return hipGetLastError();
  }
  k_start<G><<<dim3(n_start), kThreads, 0, s>>>(c, start, ws);
  for (int i = 0; i < c.steps; ++i) {
    k_product<kGram, G><<<dim3(n_square), kThreads, 0, s>>>(c, square, ws, i);
    k_product<kPoly, G><<<dim3(n_square), kThreads, 0, s>>>(c, square, ws, i);
    if (i + 1 < c.steps) k_product<kApply, G><<<dim3(n_full), kThreads, 0, s>>>(c, full, ws, i);
    else k_product<kLast, G><<<dim3(n_full), kThreads, 0, s>>>(c, full, ws, i);
  }
  return hipGetLastError();
}

}  // namespace ns
}  // namespace

int64_t ns_workspace_bytes(int count, int rows, int cols) {
  return ns::sum_bytes(count) + count * ns::place(rows, cols).size * 2;     // whole 2 KB blocks
}

hipError_t launch_ns(const NsCall& c, int dtype, void* ws, hipStream_t s) {
  return dtype == POP_F32 ? ns::run<float>(c, (char*)ws, s) : dtype == POP_BF16 ? ns::run<__bf16>(c, (char*)ws, s) : ns::run<_Float16>(c, (char*)ws, s);
}

}  // namespace pop
