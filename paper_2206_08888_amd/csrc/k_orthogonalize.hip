// Newton-Schulz orthogonalisation of stacks of matrices, and the Muon step around it (operators.h).
//
//   X = U / (|U| + eps);  steps times:  A = X X^T,  B = k1 A + k2 A A,  X = k0 X + B X
//
// with X of m x n, m <= n (matrices with more rows than columns are taken transposed).  A step multiplies X by P = k0 + B,
// and several of them may be taken in the space of A, where such polynomials are symmetric m x m matrices that commute
// (half of their tiles are computed):
//
//   A = X X^T;  per step of a segment:  Q = P Q,  A = P A P;  then X = Q X
//
// so that X, m x n, is touched twice per segment.  Errors against 64 bits, segments of 1 / 2 / 3 steps, over those of fp32
// products: 0.42 / 0.83 / 1.13 in the mean of 60 shapes from m = 65 on (ordinary gradients, the usual quintic, five steps), 0.71 /
// 4.2 / 3.0 at most, the larger ones on square matrices; of n >= 1.5 m 0.71 / 1.9 / 1.7 at most.  So results in fp32 take one step
// per segment, and results of 16 bits, whose rounding is 2e-4 or more, three where that is less work, from n = 1.5 m on
// (four 1024 x 4096: 840 us, with one step 1270; 256 x 256: 114, with one 102).  Steep steps enlarge the difference: a step
// multiplies errors of A, 2^-22 of its largest entries, by the square of its slope at 0, what is unsymmetric in them (blocks
// on the diagonal are not mirrored inside) by the third power.  Segments of three are taken while all steps together
// multiply A by at most 2^22 (kSegmentGain squared; five and six steps of the usual quintic: 2^17.8 and 2^21.4); eight of slope 5,
// 2^37, had up to 16 times the error of fp32 products, with one step less than theirs.
//
// All matrices of a call advance together, a launch per product.  Calls whose matrices all have m up to 64 take a path of
// their own: the squares of A, Q and so on fit a workgroup, and with everything in 64 bits all steps are one segment, unless they
// are too many or too steep (below, k_gram64).  (Beside larger matrices small ones cost nothing, and launches of their own would.)
//
// Products on v_mfma_f32_32x32x16_f16 from operands in two fp16 halves, x = hi + lo with 11 bits each, held in units
// (powers of two, unit_of below) that keep the largest possible entry just below 2^15, so that lo keeps its bits for
// entries down to 2^-14 of the largest: x y = hi hi + hi lo + lo hi, what is left out is below 2^-22 |x y|.  Three
// instructions in place of sixteen of the fp32 ones.  The matrix pipe rounds its accumulator after every instruction: the
// two small products have one of their own, so that a sum is rounded a third as often.
//
// Operands lie in the workspace as the instruction takes them: blocks of 32 rows x 16 contraction indices, 64 lanes
// of 8 halves (lane l: row l & 31, indices 8 (l >> 5) ..), the hi block in front of the lo block, 2 KB together,
// blocks of one row band adjacent.  Both operands have the contraction index inside, so X is kept in both orders.
#include <hip/hip_runtime.h>
#include <initializer_list>
#include <type_traits>
#include "operators.h"
#include "pop_dev.h"

namespace pop {
namespace {
namespace ns {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kPair = 1024;                 // halves of a hi and a lo block
constexpr int kSmall = 2;                   // bands of m up to which matrices can take the path in 64 bits
constexpr float kSmallGain = 0x1p20f;       // most that all steps together may multiply small singular values by there

// Where the arrays of one matrix lie, in halves from the start of its workspace.
struct Place {
  int mb, nb;                               // 32-row bands of m and n
  int64_t x, xt[2], a, b, t, q[2], size;    // X [m rows, n inside], X^T [n rows, m inside] twice; A, B, P A, Q twice
};
__host__ __device__ inline Place place(int mb, int nb) {
  Place p;
  p.mb = mb;
  p.nb = nb;
  const int64_t xs = (int64_t)mb * nb * 2 * kPair, as = (int64_t)mb * mb * 2 * kPair;
  p.x = 0; p.xt[0] = xs; p.xt[1] = 2 * xs;
  p.a = 3 * xs; p.b = p.a + as; p.t = p.b + as; p.q[0] = p.t + as; p.q[1] = p.q[0] + as;
  p.size = p.q[1] + as;
  return p;
}
__host__ __device__ inline Place place_of(int rows, int cols) {
  return place(((rows < cols ? rows : cols) + 31) / 32, ((rows < cols ? cols : rows) + 31) / 32);
}
constexpr int kSumParts = 256;              // most partial sums of one matrix's squares
__host__ __device__ inline int part_elements(int rows, int cols) {
  const int64_t n = (int64_t)rows * cols, a = (n + kSumParts - 1) / kSumParts;
  return (int)(a > 8192 ? (a + 1023) / 1024 * 1024 : 8192);
}
__host__ __device__ inline int parts(int rows, int cols) {
  const int64_t e = part_elements(rows, cols);
  return (int)(((int64_t)rows * cols + e - 1) / e);
}

// m <= 64: partial sums of X X^T over pieces of n, and Q, in squares of 16-row bands.
constexpr int kPieces = 32;                 // most pieces
__host__ __device__ inline int small_side(int m) { return (m + 15) / 16 * 16; }
__host__ __device__ inline int pieces(int n) { const int c = (n + 63) / 64; return c < kPieces ? c : kPieces; }

// Factors of a step's products (two of each product, as one may not be finite) and of what is added to them.
struct Factors { float p0, p1, old; };
struct StepFactors {
  float gram0, gram1;                       // A = X X^T
  Factors poly, q, t, next;                 // B, Q (in a segment's first step: of B and of the unit matrix), T, A
  float done0, done1;                       // X = Q X behind the step
};
// A matrix's workspace in front of its blocks.
struct Head {
  double sums[kSumParts];
  StepFactors step[POP_NS_MAX_STEPS];
};

// ---- arguments of a launch: few lines, as each is a trip to memory where it is first used

struct LayerArg {
  int per, count, mb, nb;                   // workgroups of one matrix, matrices, bands
  int64_t ws;                               // bytes to the layer's workspace
  int64_t turned;                           // more rows than columns: X is the transpose
};
struct Args {
  int first[POP_MUON_MAX_LAYERS];           // first workgroup of a layer, a multiple of 8
  int step, first_step, last_step, parity, done_parity, xt;   // number, whether the segment's first, last; which Q, Q at its end, X^T
  LayerArg layer[POP_MUON_MAX_LAYERS];
};
struct EndArg {                             // a caller's arrays of a layer
  const void* g;
  int64_t g_matrix, g_row;
  float* m;
  int64_t m_matrix, m_row;
  void* out;                                // weights, or results
  int64_t out_matrix, out_row;
  int rows, cols;
  float scale;
  int reserved;
};
struct Ends {
  const float* hparams;
  float eps;
  int nesterov;
  EndArg layer[POP_MUON_MAX_LAYERS];
};
struct NoEnds {};

// Units in front of a step of X and A = X X^T, of B = k1 A + k2 A A and of T = P A: powers of two by which entries are
// held multiplied.  No entry exceeds the largest singular value.  That of X is below `most` whatever the matrix, and
// below gain[step] |X| of the first X where eps made that small; T's are those of X times those of the next X; Q's are
// bounded by the coefficients alone.  (The limits on the exponents keep the units and what they divide finite: an X
// below 2^-100 is as good as none, and an A, B or T below 2^-60 makes no difference to X.)
__device__ inline float unit_of(float most, int limit) {
  const int e = 14 - ilogbf(fmaxf(most, 0x1p-120f));
  return ldexpf(1.0f, e < limit ? e : limit);
}
struct Bounds {                             // NsCall
  int steps, segment;
  float most, coef[POP_NS_MAX_STEPS][3], gain[POP_NS_MAX_STEPS + 1], q_most[POP_NS_MAX_STEPS];
};
__device__ inline float x_most(const Bounds& c, int step, float start) { return fminf(c.most, start * c.gain[step]); }
__device__ inline StepFactors factors_of(const Bounds& c, int k, float start) {
  const int first = k / c.segment * c.segment;
  const float k0 = c.coef[k][0], k1 = c.coef[k][1], k2 = c.coef[k][2], most = x_most(c, k, start), after = x_most(c, k + 1, start), a2 = most * most;
  const float x = unit_of(most, 100), a = unit_of(a2, 60), b = unit_of(fabsf(k1) * a2 + fabsf(k2) * a2 * a2, 60), t = unit_of(most * after, 60),
              a_next = unit_of(after * after, 60), q = unit_of(c.q_most[k], 60);
  StepFactors f;
  f.gram0 = 1.0f / x; f.gram1 = a / x;
  f.poly = {1.0f / a, k2 * (b / a), k1 * (b / a)};
  if (k == first) f.q = {q / b, 1.0f, k0 * q};
  else { const float before = unit_of(c.q_most[k - 1], 60); f.q = {1.0f / b, q / before, k0 * (q / before)}; }
  f.t = {1.0f / b, t / a, k0 * (t / a)};
  f.next = {1.0f / b, a_next / t, k0 * (a_next / t)};
  f.done0 = 1.0f / q; f.done1 = (k + 1 == c.steps ? 1.0f : unit_of(after, 100)) / unit_of(x_most(c, first, start), 100);
  return f;
}

// Workgroups go to the 8 XCDs in turn: each XCD takes an eighth of a layer's units in a row, so that its L2 reads few
// matrices, and of large ones few bands of the left operand (20 critics of 393 x 256 and
// 256 x 256, a step: 308 us with matrices dealt out to XCDs one by one, 246 so).  matrix < 0: none left.
struct At { int layer, matrix, unit; LayerArg l; };
__device__ inline At find(const Args& c) {
  const int block = (int)blockIdx.x;
  At at;
  at.layer = 0;
#pragma unroll
  for (int k = 1; k < POP_MUON_MAX_LAYERS; ++k) at.layer += block >= c.first[k];
  at.l = c.layer[at.layer];
  const int i = block - c.first[at.layer], per = at.l.per, units = per * at.l.count, n = (i & 7) * ((units + 7) / 8) + (i >> 3);
  at.matrix = n < units ? n / per : -1;
  at.unit = n % per;
  return at;
}

// a layer's workspace: the heads, then the matrices
__host__ __device__ inline int64_t head_bytes(int count) { return ((int64_t)count * sizeof(Head) + 255) / 256 * 256; }
__device__ inline Head& head_of(char* ws, const At& at) { return ((Head*)(ws + at.l.ws))[at.matrix]; }
__device__ inline _Float16* halves_of(char* ws, const At& at, const Place& p) {
  return (_Float16*)(ws + at.l.ws + head_bytes(at.l.count)) + (int64_t)at.matrix * p.size;
}

// ---- momentum and norms

constexpr int kThreads = 256;

__device__ inline double block_sum(double v, double* red) {
  for (int s = 32; s > 0; s /= 2) v += __shfl_xor(v, s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}

// The momentum's step and the sum of U's squares, a part of a matrix per workgroup; bound by memory (80 policies of 17 x 256, 256 x
// 256 and 256 x 6 in fp32: 14 us for 69 MB).
template <typename G>
__global__ void __launch_bounds__(kThreads) k_norms(Args c, Ends ends, char* ws) {
  __shared__ double red[4];
  warm_args<576>();
  const At at = find(c);
  const EndArg l = ends.layer[at.layer];
  if (at.matrix < 0) return;
  const int e = part_elements(l.rows, l.cols), n = l.rows * l.cols;
  const int lo = at.unit * e, hi = min(lo + e, n);
  const float mu = ends.hparams ? ends.hparams[3 * at.matrix + 1] : 0.0f;
  const G* g = (const G*)l.g + at.matrix * l.g_matrix;
  float* m = ends.hparams ? l.m + at.matrix * l.m_matrix : nullptr;
  // rows without gaps are one run of elements
  const bool flat = l.g_row == l.cols && (!m || l.m_row == l.cols);
  double sum = 0.0;
  // eight elements at a time: all loads ahead of the stores, which the compiler could not move them past
  const auto add = [&](float (&u)[8], float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (m) {
        v[j] = fmaf(mu, v[j], u[j]);
        u[j] = ends.nesterov ? fmaf(mu, v[j], u[j]) : v[j];
      }
      sum += (double)u[j] * u[j];
    }
  };
  if (flat && (n & 3) == 0 && (uintptr_t)g % (4 * sizeof(G)) == 0 && (uintptr_t)m % 16 == 0) {
    typedef G g4 __attribute__((ext_vector_type(4)));
    for (int i0 = lo + 4 * (int)threadIdx.x; i0 < hi; i0 += 8 * kThreads) {        // two runs of four
      const int i1 = i0 + 4 * kThreads;
      float u[8] = {}, v[8] = {};
      const g4 a = *(const g4*)(g + i0);
      f32x4 c = {}, d = {};
      g4 b = {};
      if (m) c = *(const f32x4*)(m + i0);
      if (i1 < hi) {
        b = *(const g4*)(g + i1);
        if (m) d = *(const f32x4*)(m + i1);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) { u[j] = (float)a[j]; u[4 + j] = (float)b[j]; v[j] = c[j]; v[4 + j] = d[j]; }
      add(u, v);
      if (m) {
        *(f32x4*)(m + i0) = f32x4{v[0], v[1], v[2], v[3]};
        if (i1 < hi) *(f32x4*)(m + i1) = f32x4{v[4], v[5], v[6], v[7]};
      }
    }
  } else {
    for (int i0 = lo + (int)threadIdx.x; i0 < hi; i0 += 8 * kThreads) {
      float u[8], v[8];
      int64_t to[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = i0 + j * kThreads, r = flat ? 0 : i / l.cols, k = flat ? i : i - r * l.cols;
        to[j] = r * l.m_row + k;
        u[j] = i < hi ? (float)g[r * l.g_row + k] : 0.0f;
        v[j] = m && i < hi ? m[to[j]] : 0.0f;
      }
      add(u, v);
      if (m)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (i0 + j * kThreads < hi) m[to[j]] = v[j];
    }
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) head_of(ws, at).sums[at.unit] = sum;
}

// |U| from the partial sums, the same in every workgroup
__device__ inline double norm_of(const double* sums, int n, double* red) {
  return sqrt(block_sum((int)threadIdx.x < n ? sums[threadIdx.x] : 0.0, red));
}

// ---- blocks of operands

// Accumulator tile of 32 x 32: register 4 q + r of lane l is element (row i = 8 q + 4 (l >> 5) + r, column j = l & 31).
// `put_turned` writes registers 4 q .. of it with j as the row and i inside (four i are adjacent) to turned_at() +
// turned(q); `put` with i as the row and j inside, by way of 32 x 36 words of LDS.  band: 32-row band of the target,
// inside: its 32 inner indices' number.
struct Quad { f16x4 hi, lo; };
__device__ inline Quad split(const f32x4& v) {
  Quad h;
  h.hi = __builtin_convertvector(v, f16x4);
  h.lo = __builtin_convertvector(v - __builtin_convertvector(h.hi, f32x4), f16x4);
  return h;
}
__device__ inline f32x4 value(const Quad& p) { return __builtin_convertvector(p.hi, f32x4) + __builtin_convertvector(p.lo, f32x4); }
__device__ inline int64_t pair_at(int band, int inside16, int bands_inside) { return ((int64_t)band * bands_inside * 2 + inside16) * kPair; }
__device__ inline int64_t turned_at(int band, int inside, int bands_inside) {
  const int lane = threadIdx.x & 63;
  return pair_at(band, 2 * inside, bands_inside) + ((lane & 31) * 8 + 4 * (lane >> 5));
}
__device__ constexpr int turned(int q) { return (q >> 1) * kPair + (q & 1) * 256; }
__device__ inline void put_turned(_Float16* to, const Quad& v) {
  *(f16x4*)to = v.hi;
  *(f16x4*)(to + kPair / 2) = v.lo;
}
__device__ inline Quad get_turned(const _Float16* from) { return {*(const f16x4*)from, *(const f16x4*)(from + kPair / 2)}; }
constexpr int kStride = 36;                 // words; 16-byte reads of 8 rows meet all banks
__device__ inline void stage(unsigned* scratch, int q, const Quad& v) {
  const int lane = threadIdx.x & 63;
  unsigned* to = scratch + (4 * (lane >> 5)) * kStride + (lane & 31) + 8 * q * kStride;
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 hi = __builtin_bit_cast(u32x2, v.hi), lo = __builtin_bit_cast(u32x2, v.lo);
#pragma unroll
  for (int r = 0; r < 4; ++r) to[r * kStride] = __builtin_amdgcn_perm(lo[r >> 1], hi[r >> 1], r & 1 ? 0x07060302u : 0x05040100u);
}
__device__ inline void put(_Float16* to, const unsigned* scratch, int half) {        // to: pair_at(band, 2 * inside + half, ..)
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63;
  const u32x4* from = (const u32x4*)(scratch + (lane & 31) * kStride + 16 * half + 8 * (lane >> 5));
  const u32x4 a = from[0], b = from[1];
  const u32x4 hi = {__builtin_amdgcn_perm(a[1], a[0], 0x05040100u), __builtin_amdgcn_perm(a[3], a[2], 0x05040100u),
                    __builtin_amdgcn_perm(b[1], b[0], 0x05040100u), __builtin_amdgcn_perm(b[3], b[2], 0x05040100u)};
  const u32x4 lo = {__builtin_amdgcn_perm(a[1], a[0], 0x07060302u), __builtin_amdgcn_perm(a[3], a[2], 0x07060302u),
                    __builtin_amdgcn_perm(b[1], b[0], 0x07060302u), __builtin_amdgcn_perm(b[3], b[2], 0x07060302u)};
  *(u32x4*)(to + lane * 8) = hi;
  *(u32x4*)(to + lane * 8 + kPair / 2) = lo;
}

// ---- X in both orders

// A lane's corner of block (ib, jb) of a caller's matrix; its register 4 q + r lies 8 q + r rows below.
struct Corner {
  int64_t at;                               // elements from the start of the array
  int rows;                                 // rows of the matrix from the corner on (0: the column is outside)
};
__device__ inline Corner corner(int matrix, int64_t matrix_stride, int64_t row_stride, int rows, int cols, int ib, int jb) {
  const int lane = threadIdx.x & 63, i = ib * 32 + 4 * (lane >> 5), j = jb * 32 + (lane & 31);
  return {matrix * matrix_stride + i * row_stride + j, j < cols ? max(rows - i, 0) : 0};
}

// X = U / (|U| + eps) in blocks of both orders, and the factors of all steps; bound by memory's latency (the same policies: 17 us
// for 46 MB read, 46 and the padding to whole blocks written).
template <typename G>
__global__ void __launch_bounds__(kThreads) k_start(Args c, Bounds bounds, Ends ends, char* ws) {
  __shared__ double red[4];
  __shared__ __attribute__((aligned(16))) unsigned scratch[4][32 * kStride];
  warm_args<576>();
  const At at = find(c);
  const EndArg l = ends.layer[at.layer];
  if (at.matrix < 0) return;
  const Place p = place(at.l.mb, at.l.nb);
  const float mu = ends.hparams ? ends.hparams[3 * at.matrix + 1] : 0.0f;
  const bool turned_in = l.rows > l.cols, plain = !ends.hparams || ends.nesterov;
  const int cb = turned_in ? p.mb : p.nb, wave = threadIdx.x >> 6;
  const int block = at.unit * 4 + wave;
  const bool on = block < p.mb * p.nb;
  const int ib = block / cb, jb = block % cb;
  float u[16], m[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) u[k] = m[k] = 0.0f;
  if (plain) {
    const Corner o = corner(at.matrix, l.g_matrix, l.g_row, on ? l.rows : 0, l.cols, ib, jb);
    const G* from = (const G*)l.g + o.at;
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (8 * (k >> 2) + (k & 3) < o.rows) u[k] = (float)from[(8 * (k >> 2) + (k & 3)) * l.g_row];
  }
  if (ends.hparams) {
    const Corner o = corner(at.matrix, l.m_matrix, l.m_row, on ? l.rows : 0, l.cols, ib, jb);
    const float* from = l.m + o.at;
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (8 * (k >> 2) + (k & 3) < o.rows) m[k] = from[(8 * (k >> 2) + (k & 3)) * l.m_row];
#pragma unroll
    for (int k = 0; k < 16; ++k) u[k] = plain ? fmaf(mu, m[k], u[k]) : m[k];
  }
  Head& head = head_of(ws, at);
  const double norm = norm_of(head.sums, parts(l.rows, l.cols), red), inv = 1.0 / (norm + (double)ends.eps);
  const float start = (float)(norm * inv);
  if (at.unit == 0 && (int)threadIdx.x < bounds.steps) head.step[threadIdx.x] = factors_of(bounds, threadIdx.x, start);
  const double scale = inv * unit_of(x_most(bounds, 0, start), 100);
  if (!on) return;
  _Float16* base = halves_of(ws, at, p);
  // rows of the matrix are m unless it is turned
  _Float16* across = base + (turned_in ? p.x : p.xt[0]) + turned_at(jb, ib, turned_in ? p.nb : p.mb);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f32x4 v;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = (float)((double)u[4 * q + r] * scale);
    const Quad h = split(v);
    put_turned(across + turned(q), h);
    stage(scratch[wave], q, h);
  }
  __builtin_amdgcn_wave_barrier();
  _Float16* along = base + (turned_in ? p.xt[0] : p.x) + pair_at(ib, 2 * jb, turned_in ? p.mb : p.nb);
#pragma unroll
  for (int half = 0; half < 2; ++half) put(along + half * kPair, scratch[wave], half);
}

// ---- products

__device__ inline f32x16 mfma(const f16x8& a, const f16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
// What waits for LDS only: loads stay in flight across it.
__device__ inline void sync_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
struct Pair { f16x8 hi, lo; };
__device__ inline Pair load_pair(const _Float16* p) { return {*(const f16x8*)p, *(const f16x8*)(p + kPair / 2)}; }
struct Acc {
  f32x16 large, small;
  __device__ inline void add(const Pair& l, const Pair& r) {
    small = mfma(l.hi, r.lo, small);
    large = mfma(l.hi, r.hi, large);
    small = mfma(l.lo, r.hi, small);
  }
};

// kGram: A = X X^T.  kPoly: B = k1 A + k2 A A, in the first step of a segment Q = k0 + B as well.  kMix: T = k0 A + B A
// but in the last step of a segment, Q = k0 Q + B Q but in the first.  kNext: A = k0 T + B T.  kApply: X = Q X.  kLast:
// the same, into the result.
enum { kGram = 0, kPoly = 1, kMix = 2, kNext = 3, kApply = 4, kLast = 5 };

__device__ inline void triangle(int t, int u, int& i, int& j) {       // entry u of the upper triangle of t x t tiles
  i = 0;
  while (u >= t - i) { u -= t - i; ++i; }
  j = i + u;
}
__host__ __device__ inline int tiles(int t) { return t * (t + 1) / 2; }

// One product of a launch: rows i of `left` times rows j of `right`, `inner` blocks of 16; what is added to it, k0 (kPoly:
// k1) times `old`; where the result goes with j as the row, and its mirror image (kApply: X beside X^T).
struct Product {
  const _Float16 *left, *right, *old;
  _Float16 *to, *mirror;
  int ibands, jbands, inner;
  bool turned, q_task;
};
// unit: the workgroup's number among those of its matrix; side: tiles or blocks along m.
template <int MODE> __device__ inline Product product_of(const Args& c, const At& at, const Place& p, _Float16* base, int& unit, int side) {
  Product o;
  o.turned = MODE == kLast && at.l.turned;
  o.q_task = MODE == kMix && (c.last_step || (!c.first_step && unit >= tiles(side)));
  if (MODE == kMix && unit >= tiles(side)) unit -= tiles(side);
  o.ibands = o.jbands = p.mb;
  o.inner = 2 * p.mb;
  o.old = o.to = o.mirror = nullptr;
  _Float16 *q = base + p.q[c.parity], *q_before = base + p.q[c.parity ^ 1], *done = base + p.q[c.done_parity];
  if (MODE == kGram) {
    o.left = o.right = base + p.x;
    o.to = o.mirror = base + p.a;
    o.inner = 2 * p.nb;
  } else if (MODE == kPoly) {
    o.left = o.right = o.old = base + p.a;
    o.to = o.mirror = base + p.b;
  } else if (MODE == kMix) {
    o.left = base + p.b;
    o.right = o.old = o.q_task ? q_before : base + p.a;
    o.to = o.mirror = o.q_task ? q : base + p.t;
  } else if (MODE == kNext) {
    o.left = base + p.b;
    o.right = o.old = base + p.t;
    o.to = o.mirror = base + p.a;
  } else if (o.turned) {
    o.left = base + p.xt[c.xt];
    o.right = done;
    o.ibands = p.nb;
  } else {
    o.left = done;
    o.right = base + p.xt[c.xt];
    o.jbands = p.nb;
    o.to = base + p.xt[c.xt ^ 1];
    o.mirror = base + p.x;
  }
  return o;
}
template <int MODE> __device__ inline Factors factors_of(const StepFactors& f, bool q_task) {
  if (MODE == kGram) return {f.gram0, f.gram1, 0.0f};
  if (MODE == kPoly) return f.poly;
  if (MODE == kMix) return q_task ? f.q : f.t;
  if (MODE == kNext) return f.next;
  return {f.done0, f.done1, 0.0f};
}
// The first step's Q = k0 + B, from values of B.
__device__ inline f32x4 first_q(const Factors& f, int ib, int jb, int q, const f32x4& b) {
  const int lane = threadIdx.x & 63, i = 8 * q + 4 * (lane >> 5), j = ib == jb ? lane & 31 : -1;
  f32x4 v;
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = fmaf(b[r], f.p0, i + r == j ? f.old : 0.0f);
  return v;
}

// Registers 4 q .. of a block of results: weights are read ahead of the product, written behind it.
template <int MODE, typename E> __device__ inline f32x4 read_weights(const E& ends, const At& at, int ib, int jb, int q) {
  f32x4 w = {};
  if constexpr (MODE == kLast) {
    if (ends.hparams) {
      const EndArg& l = ends.layer[at.layer];
      const Corner c = corner(at.matrix, l.out_matrix, l.out_row, l.rows, l.cols, ib, jb);
      const float* from = (const float*)l.out + c.at;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (8 * q + r < c.rows) w[r] = from[(8 * q + r) * l.out_row];
    }
  }
  return w;
}
template <typename G> __device__ inline void write_result(const Ends& ends, const At& at, int ib, int jb, int q, const f32x4& w, const f32x4& v) {
  const EndArg& l = ends.layer[at.layer];
  const Corner c = corner(at.matrix, l.out_matrix, l.out_row, l.rows, l.cols, ib, jb);
  if (ends.hparams) {
    const float* hp = ends.hparams + 3 * at.matrix;
    const float up = -hp[0] * l.scale, keep = fmaf(-hp[0], hp[2], 1.0f);
    float* to = (float*)l.out + c.at;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (8 * q + r < c.rows) to[(8 * q + r) * l.out_row] = fmaf(up, v[r], w[r] * keep);
  } else {
    G* to = (G*)l.out + c.at;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (8 * q + r < c.rows) to[(8 * q + r) * l.out_row] = (G)v[r];
  }
}

// A wavefront's block of results in both orders (mirror: or NULL).
__device__ inline void write_block(const f32x4 (&v)[4], _Float16* to, _Float16* mirror, unsigned* scratch) {
  Quad h[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    h[q] = split(v[q]);
    put_turned(to + turned(q), h[q]);
  }
  if (!mirror) return;
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int q = 0; q < 4; ++q) stage(scratch, q, h[q]);
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int half = 0; half < 2; ++half) put(mirror + half * kPair, scratch, half);
  __builtin_amdgcn_wave_barrier();
}

// One 32 x 32 block per workgroup; the wavefronts take a quarter of the contraction each, then a quarter of the block.  Bound
// by latency (arguments, matrix head, operands, LDS, results: ten of 256 x 256, X X^T 5.3 us, B 5.7, of which 1 is matrix
// time); a launch's gap is another 1 to 2 us.
template <int MODE, typename G, typename E>
__global__ void __launch_bounds__(kThreads) k_block(Args c, E ends, char* ws) {
  __shared__ float part[4][16][64];
  __shared__ __attribute__((aligned(16))) unsigned scratch[32 * kStride];
  warm_args<sizeof(Args) + (std::is_same<E, Ends>::value ? 256 : 0)>();
  const At at = find(c);
  if (at.matrix < 0) return;
  const Place p = place(at.l.mb, at.l.nb);
  _Float16* base = halves_of(ws, at, p);
  int unit = at.unit, ib, jb;
  const Product o = product_of<MODE>(c, at, p, base, unit, p.mb);
  if (MODE < kApply) triangle(p.mb, unit, ib, jb);
  else { ib = unit / o.jbands; jb = unit - ib * o.jbands; }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int q4 = (o.inner + 3) / 4, lo = wave * q4, hi = min(lo + q4, o.inner);
  const _Float16 *lp = o.left + (int64_t)ib * o.inner * kPair + lane * 8, *rp = o.right + (int64_t)jb * o.inner * kPair + lane * 8;
  Acc acc = {};
  int k = lo;
  const StepFactors& step = head_of(ws, at).step[c.step];
  const Factors f = factors_of<MODE>(step, o.q_task), fq = step.q;
  const int64_t place_to = turned_at(jb, ib, p.mb) + turned(wave);
  Quad old = {};
  if (o.old) old = get_turned(o.old + place_to);
  const f32x4 weights = read_weights<MODE>(ends, at, ib, jb, wave);
  for (; k + 4 <= hi; k += 4) {
    Pair x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = load_pair(lp + (int64_t)(k + i) * kPair); y[i] = load_pair(rp + (int64_t)(k + i) * kPair); }
#pragma unroll
    for (int i = 0; i < 4; ++i) acc.add(x[i], y[i]);
  }
  for (; k < hi; ++k) acc.add(load_pair(lp + (int64_t)k * kPair), load_pair(rp + (int64_t)k * kPair));
#pragma unroll
  for (int i = 0; i < 16; ++i) part[wave][i][lane] = acc.large[i] + acc.small[i];
  __syncthreads();
  const f32x4 before = value(old);
  f32x4 v;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = 4 * wave + r;
    v[r] = ((part[0][i][lane] + part[1][i][lane]) + (part[2][i][lane] + part[3][i][lane])) * f.p0 * f.p1 + before[r] * f.old;
  }
  if constexpr (MODE == kLast) {
    write_result<G>(ends, at, ib, jb, wave, weights, v);
  } else {
    const bool mirrored = MODE == kApply || ib != jb, q_alone = MODE == kPoly && c.first_step && c.last_step;
    const int64_t mirror_to = pair_at(ib, 2 * jb + wave, MODE == kApply ? p.nb : p.mb);
    const auto write = [&](_Float16* to, _Float16* mirror) {
      const Quad h = split(v);
      put_turned(to + place_to, h);
      if (!mirrored) return;
      __syncthreads();                        // (of a block before)
      stage(scratch, wave, h);
      __syncthreads();
      if (wave < 2) put(mirror + mirror_to, scratch, wave);
    };
    if (!q_alone) write(o.to, o.mirror);
    if (MODE == kPoly && c.first_step) {
      v = first_q(fq, ib, jb, wave, v);
      write(base + p.q[0], base + p.q[0]);
    }
  }
}

// kMix and kApply: tiles of 64 x 64, a block per wavefront, operands straight from the caches into registers, four blocks of
// the contraction ahead.  Bound by latency as k_block, with half of its traffic: ten of 256 x 256, X = Q X 8.1 us.
constexpr int kQuad = 2;                    // bands of a tile's side
template <int MODE, typename G, typename E>
__global__ void __launch_bounds__(kThreads) k_quad(Args c, E ends, char* ws) {
  __shared__ __attribute__((aligned(16))) unsigned all_scratch[4][32 * kStride];
  warm_args<sizeof(Args) + (std::is_same<E, Ends>::value ? 256 : 0)>();
  const At at = find(c);
  if (at.matrix < 0) return;
  const Place p = place(at.l.mb, at.l.nb);
  _Float16* base = halves_of(ws, at, p);
  const int side = (p.mb + kQuad - 1) / kQuad;
  int unit = at.unit, ti, tj;
  const Product o = product_of<MODE>(c, at, p, base, unit, side);
  if (MODE < kApply) {
    triangle(side, unit, ti, tj);
  } else {
    const int jt = (o.jbands + kQuad - 1) / kQuad;
    ti = unit / jt;
    tj = unit - ti * jt;
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, ib = ti * kQuad + (wave >> 1), jb = tj * kQuad + (wave & 1);
  if (ib >= o.ibands || jb >= o.jbands) return;
  const _Float16 *lp = o.left + (int64_t)ib * o.inner * kPair + lane * 8, *rp = o.right + (int64_t)jb * o.inner * kPair + lane * 8;
  struct Batch { Pair x[4], y[4]; } ahead[2];
  // (behind the end the last blocks are read again, and not used: no conditions, as in k_tile)
  const auto fetch = [&](Batch& b, int k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t at_k = (int64_t)min(k + i, o.inner - 1) * kPair;
      b.x[i] = load_pair(lp + at_k);
      b.y[i] = load_pair(rp + at_k);
    }
  };
  Acc acc = {};
  const auto multiply = [&](const Batch& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc.add(b.x[i], b.y[i]);
  };
  fetch(ahead[0], 0);
  fetch(ahead[1], 4);
  const StepFactors& step = head_of(ws, at).step[c.step];
  const Factors f = factors_of<MODE>(step, o.q_task);
  const int64_t place_to = turned_at(jb, ib, p.mb), mirror_to = pair_at(ib, 2 * jb, MODE == kApply ? p.nb : p.mb);
  Quad old[4] = {};
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (MODE == kMix) old[q] = get_turned(o.old + place_to + turned(q));
  const int whole = o.inner / 8 * 8;
  for (int k = 0; k < whole; k += 8) {
    multiply(ahead[0]);
    fetch(ahead[0], k + 8);
    multiply(ahead[1]);
    fetch(ahead[1], k + 12);
  }
  if (o.inner & 4) {
    multiply(ahead[0]);
    ahead[0] = ahead[1];
  }
  if (o.inner & 2) {                          // `inner` is even
    acc.add(ahead[0].x[0], ahead[0].y[0]);
    acc.add(ahead[0].x[1], ahead[0].y[1]);
  }
  f32x4 v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const f32x4 before = value(old[q]);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[q][r] = (acc.large[4 * q + r] + acc.small[4 * q + r]) * f.p0 * f.p1 + before[r] * f.old;
  }
  const bool mirrored = MODE == kApply || ti != tj;
  write_block(v, o.to + place_to, mirrored ? o.mirror + mirror_to : nullptr, all_scratch[wave]);
}

// Tiles of 128 x 64 BJ, 64 x 32 BJ per wavefront, 32 contraction indices at a time.  The right operand goes through LDS, the
// left one, which two wavefronts share, straight into registers.  The next stage is on its way in registers.  With 2048 x
// 2048 matrices 128 x 128 tiles run at 840 TFLOP/s of fp16 products, prologue and epilogue included, where a large fp16
// product of the library reaches 1130.  Four of 1024 x 4096: X = Q X 127 us, 815 TFLOP/s; X X^T 100, 580, and
// squares of A 31, 470, as 288 half tiles on 256 CUs leave some with two.  Products of 256 x 256 (80 of them:
// as halves X X^T 16, B 16, whole X 25) are short of stages, eight, beside their prologue and epilogue.  Eight wavefronts with both operands
// in LDS: the same time; four wavefronts so: 395 against 358 us a step of 80 agents.
//
// Halves of tiles on the diagonal: the left one's lower blocks are the right one's upper blocks mirrored and are not
// computed.  Such light halves are dealt out last, as those are the workgroups that share a CU with another: four of 1024 x
// 1024, 256 heavy halves and 32 light ones on 256 CUs: squares 34.2 us with all halves alike, 31.3 so, X X^T over 4096 111 and
// 100.
constexpr int kTile = 4, kTileThreads = 256;
// The task, tile, half (and at.matrix) of a workgroup: an eighth of the heavy halves per XCD, behind them an eighth of the light ones.
__device__ inline int light_last(const Args& c, At& at, int side, int& ti, int& tj, int& half) {
  const int tasks = at.l.per / (2 * tiles(side)), light = tasks * side, heavy = at.l.per - light;
  const int i = (int)blockIdx.x - c.first[at.layer], rank = i >> 3, before = (heavy * at.l.count + 7) / 8;
  const bool is_heavy = rank < before;
  const int per = is_heavy ? heavy : light, total = per * at.l.count;
  const int n = is_heavy ? (i & 7) * before + rank : (i & 7) * ((total + 7) / 8) + rank - before;
  at.matrix = n < total && (is_heavy || rank - before < (total + 7) / 8) ? n / per : -1;
  int u = n % per;
  const int task = u / (per / tasks);
  u -= task * (per / tasks);
  if (is_heavy) {
    ti = 0;
    while (u >= 2 * (side - ti) - 1) { u -= 2 * (side - ti) - 1; ++ti; }
    tj = ti + (u + 1) / 2;
    half = (u + 1) & 1;
  } else {
    ti = tj = u;
    half = 0;
  }
  return task;
}
template <int MODE, typename G, typename E, int BJ>
__global__ void __launch_bounds__(kTileThreads, 2) k_tile(Args c, E ends, char* ws) {
  __shared__ __attribute__((aligned(16))) _Float16 staged[2][2 * BJ * 2 * kPair];
  __shared__ __attribute__((aligned(16))) unsigned all_scratch[4][32 * kStride];
  warm_args<sizeof(Args) + (std::is_same<E, Ends>::value ? 256 : 0)>();
  At at = find(c);
  const Place p = place(at.l.mb, at.l.nb);
  const int side = (p.mb + kTile - 1) / kTile;
  int unit = BJ == 2 ? at.unit : at.unit >> 1, ti, tj;         // a tile of 128 x 128, and which half of it
  int half_of = BJ == 2 ? 0 : at.unit & 1;
  if (BJ == 1 && MODE < kApply) unit = light_last(c, at, side, ti, tj, half_of) * tiles(side);
  if (at.matrix < 0) return;
  _Float16* base = halves_of(ws, at, p);
  const Product o = product_of<MODE>(c, at, p, base, unit, side);
  if (MODE < kApply) {
    if (BJ == 2) triangle(side, unit, ti, tj);
  } else {
    const int jt = (o.jbands + kTile - 1) / kTile;
    ti = unit / jt;
    tj = unit - ti * jt;
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wi = wave >> 1, wj = wave & 1;
  const int ib0 = ti * kTile + 2 * wi, j_first = tj * kTile + 2 * half_of, jb0 = j_first + BJ * wj, stages = o.inner / 2;
  // (a band beyond the edge: the last one again, its results are not stored; behind the last stage it is read again:
  // without conditions a wait for one stage's loads leaves those of the next in flight)
  const _Float16* lp[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) lp[b] = o.left + (int64_t)min(ib0 + b, o.ibands - 1) * o.inner * kPair + lane * 8;
  if (j_first >= o.jbands) return;
  // this wavefront brings one of the right bands, or with two of them a half of one
  const _Float16* rp = o.right + (int64_t)min(j_first + (BJ == 2 ? wave : wave >> 1), o.jbands - 1) * o.inner * kPair +
                       (BJ == 2 ? 0 : (wave & 1) * kPair) + lane * 8;
  struct Left { Pair v[2][2]; } left[2];
  struct Way { f16x8 v[2 * BJ]; } way;
  const auto fetch_left = [&](Left& l, int stage) {
    const int64_t off = (int64_t)min(stage, stages - 1) * 2 * kPair;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int k = 0; k < 2; ++k) l.v[b][k] = load_pair(lp[b] + off + k * kPair);
  };
  const auto fetch_right = [&](int stage) {
    const _Float16* from = rp + (int64_t)min(stage, stages - 1) * 2 * kPair;
#pragma unroll
    for (int i = 0; i < 2 * BJ; ++i) way.v[i] = *(const f16x8*)(from + i * (kPair / 2));
  };
  const auto land = [&](int half) {
#pragma unroll
    for (int i = 0; i < 2 * BJ; ++i) *(f16x8*)&staged[half][wave * BJ * kPair + i * (kPair / 2) + lane * 8] = way.v[i];
  };
  Acc acc[2][BJ] = {};
  const auto multiply = [&](int half, const Left& l) {
    const _Float16* here = staged[half] + lane * 8;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < BJ; ++j) {
        const Pair y = load_pair(here + ((BJ * wj + j) * 2 + k) * kPair);
#pragma unroll
        for (int b = 0; b < 2; ++b) acc[b][j].add(l.v[b][k], y);
      }
  };
  fetch_right(0);
  fetch_left(left[0], 0);
  land(0);
  fetch_right(1);
  const StepFactors& step = head_of(ws, at).step[c.step];
  const Factors f = factors_of<MODE>(step, o.q_task), fq = step.q;
  sync_lds();
  if (BJ == 1 && MODE < kApply && ti == tj && half_of == 0 && __builtin_amdgcn_readfirstlane(wi)) {
    for (int g = 0; g < (stages & ~1); ++g) {                  // below the diagonal: only the right operand is brought
      land((g & 1) ^ 1);
      fetch_right(g + 2);
      sync_lds();
    }
    return;
  }
  // a stage: its right operand is in LDS half `half`, its left one in `now`; the next ones on their way
  const auto stage_of = [&](int g, int half, const Left& now, Left& next) {
    fetch_left(next, g + 1);
    multiply(half, now);
    land(half ^ 1);
    fetch_right(g + 2);
    sync_lds();
  };
  for (int g = 0; g + 1 < stages; g += 2) {
    stage_of(g, 0, left[0], left[1]);
    stage_of(g + 1, 1, left[1], left[0]);
  }
  if (stages & 1) multiply(0, left[0]);
  unsigned* scratch = all_scratch[wave];
  const bool mirrored = MODE == kApply || (MODE < kApply && (ti != tj || (BJ == 1 && half_of == 1 && wi == 0)));
#pragma unroll
  for (int bi = 0; bi < 2; ++bi)
#pragma unroll
    for (int bj = 0; bj < BJ; ++bj) {
      const int ib = ib0 + bi, jb = jb0 + bj;
      if (ib >= o.ibands || jb >= o.jbands) continue;
      const int64_t place_to = turned_at(jb, ib, p.mb), mirror_to = pair_at(ib, 2 * jb, MODE == kApply ? p.nb : p.mb);
      Quad old[4] = {};
      f32x4 v[4], weights[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (MODE == kPoly || MODE == kMix || MODE == kNext) old[q] = get_turned(o.old + place_to + turned(q));
        weights[q] = read_weights<MODE>(ends, at, ib, jb, q);
      }
      const Acc& sum = acc[bi][bj];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 before = value(old[q]);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[q][r] = (sum.large[4 * q + r] + sum.small[4 * q + r]) * f.p0 * f.p1 + before[r] * f.old;
      }
      if constexpr (MODE == kLast) {
#pragma unroll
        for (int q = 0; q < 4; ++q) write_result<G>(ends, at, ib, jb, q, weights[q], v[q]);
      } else {
        if (!(MODE == kPoly && c.first_step && c.last_step))        // a segment of one step: only Q is used
          write_block(v, o.to + place_to, mirrored ? o.mirror + mirror_to : nullptr, scratch);
        if (MODE == kPoly && c.first_step) {
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = first_q(fq, ib, jb, q, v[q]);
          write_block(v, base + p.q[0] + place_to, mirrored ? base + p.q[0] + mirror_to : nullptr, scratch);
        }
      }
    }
}

// ---- m <= 64, in 64 bits

// The 64-bit path: k_gram64 updates the momentum and sums U U^T over a piece of n, k_square64 adds the pieces up (the trace
// is |U|^2), takes all steps as Q of U U^T / (|U| + eps)^2, and k_last64 multiplies Q by U.  Three launches, in which k_square64's
// products, one after the other in one workgroup per matrix, are the longest part: 8 of 17 x 2000 31 us (48 as fp16 halves
// in segments of three), 6 of 3 x 740 21 (44), 8 of 64 x 2048 80 (58).  That part on vector instructions made it 119, on the
// matrix ones with a wavefront's tiles one by one 159, its chains interleaved 92, from eight wavefronts 77, with tiles on
// the diagonal mirrored 80.
//
// What rounding makes of an eigenvalue of zero, about 2^-53 of either sign, grows with every step as small eigenvalues do.
// Large, it is an error of its size; far below zero, steps diverge.  So the path is taken while all steps together multiply
// eigenvalues by at most 2^40 (kSmallGain squared; eleven steps of the usual quintic: 2^39.3), which leaves 2^-13 of the largest.
// Up to there errors are the result's rounding or little more (6 x 256 of rank 3, eleven steps: 4e-8, products in 32 bits 1e-2);
// beyond it, in emulation, 14 steps 8e-3, 16 steps 5.  More or steeper steps take the general path.

constexpr int kChunk = 64, kChunkStride = 65;
// U's columns (of X) j0 .. j0 + 63 to LDS, zeros outside; `update`: with the momentum's step.
template <typename G> __device__ inline void load_chunk(const Ends& ends, const EndArg& l, int matrix, bool update, int j0, float (*x)[kChunkStride]) {
  const bool turned_in = l.rows > l.cols;
  const int m = turned_in ? l.cols : l.rows, n = turned_in ? l.rows : l.cols, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float mu = ends.hparams ? ends.hparams[3 * matrix + 1] : 0.0f;
  const G* g = (const G*)l.g + matrix * l.g_matrix;
  float* mom = ends.hparams ? l.m + matrix * l.m_matrix : nullptr;
  float u[16], v[16];
  // lanes along the caller's columns, four rows at a time: rows and columns of this chunk
  const int c0 = turned_in ? 0 : j0, r0 = turned_in ? j0 : 0, rows = turned_in ? min(n - j0, 64) : m, cols = turned_in ? m : min(n - j0, 64);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int r = wave + 4 * k;
    const bool in = r < rows && lane < cols;
    u[k] = in ? (float)g[(r0 + r) * l.g_row + c0 + lane] : 0.0f;
    v[k] = in && mom ? mom[(r0 + r) * l.m_row + c0 + lane] : 0.0f;
  }
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int r = wave + 4 * k;
    if (mom) {
      if (update) {
        v[k] = fmaf(mu, v[k], u[k]);
        if (r < rows && lane < cols) mom[(r0 + r) * l.m_row + c0 + lane] = v[k];
      }
      u[k] = ends.nesterov ? fmaf(mu, v[k], u[k]) : v[k];
    }
    if (turned_in) x[lane][r] = u[k];
    else x[r][lane] = u[k];
  }
}

struct Small { double *piece, *q; int side; };     // piece: [pieces, side, side]
__device__ inline Small small_of(char* ws, const At& at, const EndArg& l) {
  const int m = min(l.rows, l.cols), n = max(l.rows, l.cols), side = small_side(m);
  double* base = (double*)(ws + at.l.ws + head_bytes(at.l.count)) + (int64_t)at.matrix * (pieces(n) + 1) * side * side;
  return {base, base + (int64_t)pieces(n) * side * side, side};
}

// Squares of up to 4 x 4 tiles on v_mfma_f64_16x16x4_f64: lane l supplies row (column) l & 15 of index l >> 4, and register r of
// the result is element (4 r + (l >> 4), l & 15) of the tile.  The tiles on and above the diagonal go round the wavefronts, at
// most three to each.
typedef double f64x4 __attribute__((ext_vector_type(4)));
constexpr int kMine = 3;
struct Tiles { int i[kMine], j[kMine], n; };
// Tiles `wave`, `wave` + waves, .. of `count` times the triangle.
__device__ inline Tiles tiles_of(int side, int waves, int count) {
  const int t = side / 16, wave = threadIdx.x >> 6, per = tiles(t);
  Tiles m = {};
#pragma unroll
  for (int s = 0; s < kMine; ++s) {
    const int u = wave + s * waves;
    if (u < count * per) {
      triangle(t, u % per, m.i[s], m.j[s]);
      ++m.n;
    }
  }
  return m;
}

template <typename G>
__global__ void __launch_bounds__(kThreads) k_gram64(Args c, Ends ends, char* ws) {
  __shared__ float x[64][kChunkStride];
  warm_args<576>();
  const At at = find(c);
  if (at.matrix < 0) return;
  const EndArg l = ends.layer[at.layer];
  const Small w = small_of(ws, at, l);
  const int n = max(l.rows, l.cols), chunks = (n + kChunk - 1) / kChunk, parts = pieces(n), lane = threadIdx.x & 63;
  const Tiles mine = tiles_of(w.side, 4, 1);
  f64x4 acc[kMine] = {};
  for (int p = at.unit; p < chunks; p += parts) {
    __syncthreads();
    load_chunk<G>(ends, l, at.matrix, true, p * kChunk, x);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kMine; ++t) {
      if (t >= mine.n) break;
      const float *a = &x[16 * mine.i[t] + (lane & 15)][lane >> 4], *b = &x[16 * mine.j[t] + (lane & 15)][lane >> 4];
#pragma unroll
      for (int k = 0; k < kChunk; k += 4) acc[t] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)a[k], (double)b[k], acc[t], 0, 0, 0);
    }
  }
  double* to = w.piece + (int64_t)at.unit * w.side * w.side;
#pragma unroll
  for (int t = 0; t < kMine; ++t) {
    if (t >= mine.n) break;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * mine.i[t] + 4 * r + (lane >> 4), j = 16 * mine.j[t] + (lane & 15);
      to[i * w.side + j] = acc[t][r];
      if (mine.i[t] != mine.j[t]) to[j * w.side + i] = acc[t][r];
    }
  }
}

struct Coefs { int steps; float eps, coef[POP_NS_MAX_STEPS][3]; };
constexpr int kSquareStride = 72;           // doubles of an LDS row: four rows of 16 meet every bank twice
constexpr int kSquareThreads = 512;
__global__ void __launch_bounds__(kSquareThreads) k_square64(Args c, Ends ends, Coefs coefs, char* ws) {
  __shared__ double A[64 * kSquareStride], B[64 * kSquareStride], Q[64 * kSquareStride];
  warm_args<576>();
  const At at = find(c);
  if (at.matrix < 0) return;
  const EndArg l = ends.layer[at.layer];
  const Small w = small_of(ws, at, l);
  const int parts = pieces(max(l.rows, l.cols)), side = w.side, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = kSquareThreads / 64;
  const auto element = [](int i, int j) { return i * kSquareStride + j; };
  for (int e = threadIdx.x; e < side * side; e += kSquareThreads) {
    double v = 0.0;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) v += w.piece[(int64_t)p * side * side + e];
    A[element(e / side, e % side)] = v;
  }
  __syncthreads();
  double norm2 = 0.0;
  for (int i = 0; i < side; ++i) norm2 += A[element(i, i)];
  const double inv = 1.0 / (sqrt(norm2) + (double)coefs.eps);
  __syncthreads();
  for (int e = threadIdx.x; e < side * side; e += kSquareThreads) {
    A[element(e / side, e % side)] *= inv * inv;
    Q[element(e / side, e % side)] = e / side == e % side ? 1.0 : 0.0;
  }
  __syncthreads();
  // A product of two of the (symmetric) squares, tile by tile: f * left * right + g * old, in both triangles of `to`, which may
  // be `old` or an operand (behind the barrier all have read it).  Elements above the diagonal stand for those below it on
  // the diagonal's tiles too: what makes A and Q unsymmetric grows by a step's slope to the third, not to the second (with those
  // tiles as they are computed, 6 x 256 of rank 3, nine steps 2e-4, eleven 0.3).  A wavefront's tiles take turns, so that no
  // instruction waits for the one before it, with the operands of 16 indices read ahead of them.
  struct Task { const double *left, *right, *old; double *to, f, g; };
  const auto phase = [&](const Tiles& mine, const Task (&task)[kMine]) {
    f64x4 v[kMine];
    const double *a[kMine], *b[kMine];
#pragma unroll
    for (int t = 0; t < kMine; ++t) {
      v[t] = f64x4{};
      a[t] = task[t].left + element(lane >> 4, 16 * mine.i[t] + (lane & 15));
      b[t] = task[t].right + element(lane >> 4, 16 * mine.j[t] + (lane & 15));
    }
    const auto over = [&](auto count) {
      for (int k = 0; k < side; k += 16) {
        double x[kMine][4], y[kMine][4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int t = 0; t < decltype(count)::value; ++t) {
            x[t][q] = a[t][(k + 4 * q) * kSquareStride];
            y[t][q] = b[t][(k + 4 * q) * kSquareStride];
          }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int t = 0; t < decltype(count)::value; ++t) v[t] = __builtin_amdgcn_mfma_f64_16x16x4f64(x[t][q], y[t][q], v[t], 0, 0, 0);
      }
#pragma unroll
      for (int t = 0; t < decltype(count)::value; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          v[t][r] = task[t].f * v[t][r] + task[t].g * task[t].old[element(16 * mine.i[t] + 4 * r + (lane >> 4), 16 * mine.j[t] + (lane & 15))];
    };
    if (mine.n == 3) over(std::integral_constant<int, 3>());
    else if (mine.n == 2) over(std::integral_constant<int, 2>());
    else if (mine.n == 1) over(std::integral_constant<int, 1>());
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kMine; ++t)
      if (t < mine.n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int i = 16 * mine.i[t] + 4 * r + (lane >> 4), j = 16 * mine.j[t] + (lane & 15);
          if (i > j) continue;
          task[t].to[element(i, j)] = v[t][r];
          task[t].to[element(j, i)] = v[t][r];
        }
    __syncthreads();
  };
  const int per = tiles(side / 16);
  const Tiles one = tiles_of(side, waves, 1), two = tiles_of(side, waves, 2);
  for (int k = 0; k < coefs.steps; ++k) {
    const double k0 = coefs.coef[k][0], k1 = coefs.coef[k][1], k2 = coefs.coef[k][2];
    const Task poly = {A, A, A, B, k2, k1}, q = {B, Q, Q, Q, 1.0, k0}, next = {B, A, A, A, 1.0, k0};
    phase(one, {poly, poly, poly});
    if (k + 1 == coefs.steps) {
      phase(one, {q, q, q});
      break;
    }
    Task both[kMine];                       // Q = P Q, and A = P A of the second triangle
#pragma unroll
    for (int s = 0; s < kMine; ++s) both[s] = wave + s * waves < per ? q : next;
    phase(two, both);
    phase(one, {next, next, next});         // A = P P A
  }
  for (int e = threadIdx.x; e < side * side; e += kSquareThreads) w.q[e] = Q[element(e / side, e % side)] * inv;
}

// Q U for 64 columns of X; Q has 1 / (|U| + eps) in it.
template <typename G>
__global__ void __launch_bounds__(kThreads) k_last64(Args c, Ends ends, char* ws) {
  __shared__ float x[64][kChunkStride];
  __shared__ double q[64 * 64];
  warm_args<576>();
  const At at = find(c);
  if (at.matrix < 0) return;
  const EndArg l = ends.layer[at.layer];
  const Small w = small_of(ws, at, l);
  const bool turned_in = l.rows > l.cols;
  const int m = min(l.rows, l.cols), n = max(l.rows, l.cols), j0 = at.unit * kChunk, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  load_chunk<G>(ends, l, at.matrix, false, j0, x);
  for (int e = threadIdx.x; e < w.side * w.side; e += kThreads) q[e] = w.q[e];
  __syncthreads();
  const float* hp = ends.hparams ? ends.hparams + 3 * at.matrix : nullptr;
  const float up = hp ? -hp[0] * l.scale : 0.0f, keep = hp ? fmaf(-hp[0], hp[2], 1.0f) : 0.0f;
  // lanes along the caller's columns: an element of row r and column `col` of its matrix
  const int rows = turned_in ? min(n - j0, 64) : m, cols = turned_in ? m : min(n - j0, 64), r0 = turned_in ? j0 : 0, c0 = turned_in ? 0 : j0;
  // and of sixteen rows per wavefront
  const int first = wave * 16;
  if (first >= rows) return;
  double v[16] = {};
  if (turned_in) {
    for (int k = 0; k < m; ++k) {
      const double a = q[k * w.side + min(lane, w.side - 1)];
#pragma unroll
      for (int r = 0; r < 16; ++r) v[r] = fma(a, (double)x[k][first + r], v[r]);
    }
  } else {
    for (int k = 0; k < m; ++k) {
      const double a = x[k][lane];
      const double* b = q + k * w.side + first;             // first < m, and the side is a multiple of 16
#pragma unroll
      for (int r = 0; r < 16; ++r) v[r] = fma(a, b[r], v[r]);
    }
  }
  if (lane >= cols) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if (first + r >= rows) break;
    const int64_t to = at.matrix * l.out_matrix + (int64_t)(r0 + first + r) * l.out_row + c0 + lane;
    if (hp) ((float*)l.out)[to] = fmaf(up, (float)v[r], ((const float*)l.out)[to] * keep);
    else ((G*)l.out)[to] = (G)(float)v[r];
  }
}

// no steps: X itself
template <typename G>
__global__ void __launch_bounds__(kThreads) k_no_steps(Args c, Ends ends, char* ws) {
  __shared__ double red[4];
  warm_args<576>();
  const At at = find(c);
  const EndArg l = ends.layer[at.layer];
  if (at.matrix < 0) return;
  const float inv = (float)(1.0 / (norm_of(head_of(ws, at).sums, parts(l.rows, l.cols), red) + (double)ends.eps));
  const int e = part_elements(l.rows, l.cols), n = l.rows * l.cols;
  const int lo = at.unit * e, hi = min(lo + e, n);
  const float* hp = ends.hparams ? ends.hparams + 3 * at.matrix : nullptr;
  for (int i = lo + (int)threadIdx.x; i < hi; i += kThreads) {
    const int r = i / l.cols, k = i - r * l.cols;
    const float g = (float)((const G*)l.g)[at.matrix * l.g_matrix + r * l.g_row + k];
    if (hp) {
      const float m = l.m[at.matrix * l.m_matrix + r * l.m_row + k], u = ends.nesterov ? fmaf(hp[1], m, g) : m;
      float* to = (float*)l.out + at.matrix * l.out_matrix + r * l.out_row + k;
      *to = fmaf(-hp[0] * l.scale, u * inv, *to * fmaf(-hp[0], hp[2], 1.0f));
    } else {
      ((G*)l.out)[at.matrix * l.out_matrix + r * l.out_row + k] = (G)(g * inv);
    }
  }
}

// ---- launches

// Fills in a launch's workgroups, `per(layer, place)` for each matrix and `spare` (a multiple of 8) for each layer; returns their
// number.
template <typename F> int lay_out(const NsCall& c, Args& a, int spare, F per) {
  int64_t off = 0;
  int blocks = 0;
  for (int k = 0; k < POP_MUON_MAX_LAYERS; ++k) {
    a.first[k] = k < c.n_layers ? blocks : 0x7fffffff;
    a.layer[k] = LayerArg{};
    if (k >= c.n_layers) continue;
    const NsLayer& l = c.layer[k];
    const Place p = place_of(l.rows, l.cols);
    a.layer[k] = {per(l, p), l.count, p.mb, p.nb, off, l.rows > l.cols};
    blocks += (l.count * a.layer[k].per + 7) / 8 * 8 + (a.layer[k].per ? spare : 0);
    off += ns_workspace_bytes(l.count, l.rows, l.cols);
  }
  // a layer without workgroups starts where the next one does, and is passed over
  return blocks;
}

Args args_of(int step, int first, int last, int xt) {
  Args a = {};
  a.step = step;
  a.first_step = step == first; a.last_step = step == last;
  a.parity = (step - first) & 1; a.done_parity = (last - first) & 1;
  a.xt = xt;
  return a;
}

// Which kernel a product takes, by the 128 x 128 tiles of the whole launch (us: k_tile of 128 x 128 / of 128 x 64 / k_quad
// for kMix and kApply, else k_block; light halves as heavy ones).  256 x 256 matrices, X X^T of 8: 11.0 / 7.3 / 4.7, 20: 11.8 / 8.9 / 6.5, 40: 12.7 / 10.0
// / 9.7, 80: 14.8 / 14.5 / 15.8, 160: 24.3 / 27.0 / 28.5; X = Q X of 20: 13.3 / 10.2 / 12.4, 40: 14.2 / 14.6 / 16.2, 80: 23.0 /
// 21.5 / 27.6; four of 1024 x 4096: X X^T 108 / 113 / 120, X = Q X 127 / 150 / 223; one of 2048 x 2048: 54 / 58 / 73.
// Triangles, whose light halves come last, keep halves up to 400 tiles (all steps of fp32 calls, 128 x 128 / halves): 272 tiles
// (two of 2048 x 2048) 1445 / 1314, 288 (eight of 1024 x 1024) 794 / 732, 300 (100 of 256 x 256) 335 / 304, 390 (130) 402 / 398; of
// 400, 40 of 512 x 512 661 / 663, 40 of 400 x 640 588 / 578, 80 policies of 17 x 256, 256 x 256 and 256 x 6 332 / 315.  Beyond, either is
// ahead by up to 5 %, as the last workgroups fill the CUs: 408 (three of 2048 x 2048) 1792 / 1876, 432 (twelve of 1024 x 1024) 1014 /
// 1044, 500 (50 of 512 x 512) 774 / 792, 600 (60) 925 / 884, 800 (80) 1186 / 1205, 500 (100 policies) 404 / 376; from 1000 on whole
// tiles: 1008 (28 of 1024 x 1024) 2397 / 2510, 1200 (400 of 256 x 256) 1177 / 1216, 1280 (256 policies) 936 / 975.
constexpr int kTilesFrom = 256, kTrianglesFrom = 401, kHalvesFrom = 128, kQuadsFrom = 128;

template <int MODE, typename G, typename E, typename N>
void launch_product(const NsCall& c, Args a, const E& ends, char* ws, hipStream_t stream, N count) {
  const auto with = [&](int side, int halves) {
    // (two kinds of halves, each dealt out by eighths)
    return lay_out(c, a, halves == 2 && MODE < kApply ? 8 : 0, [&](const NsLayer&, const Place& p) { return halves * count(p, (p.mb + side - 1) / side, (p.nb + side - 1) / side); });
  };
  int blocks = with(kTile, 1);
  if (blocks == 0) return;
  if (blocks >= (MODE < kApply ? kTrianglesFrom : kTilesFrom)) {
    k_tile<MODE, G, E, 2><<<dim3(blocks), kTileThreads, 0, stream>>>(a, ends, ws);
    return;
  }
  if (blocks >= kHalvesFrom) {
    blocks = with(kTile, 2);
    k_tile<MODE, G, E, 1><<<dim3(blocks), kTileThreads, 0, stream>>>(a, ends, ws);
    return;
  }
  if constexpr (MODE == kMix || MODE == kApply) {
    blocks = with(kQuad, 1);
    if (blocks >= kQuadsFrom && (MODE == kApply || !(a.first_step || a.last_step))) {
      k_quad<MODE, G><<<dim3(blocks), kThreads, 0, stream>>>(a, ends, ws);
      return;
    }
  }
  blocks = with(1, 1);
  k_block<MODE, G><<<dim3(blocks), kThreads, 0, stream>>>(a, ends, ws);
}

template <typename G> hipError_t run(const NsCall& c, char* ws, hipStream_t stream) {
  Ends ends = {};
  ends.hparams = c.hparams;
  ends.eps = c.eps;
  ends.nesterov = c.nesterov;
  for (int k = 0; k < c.n_layers; ++k) {
    const NsLayer& l = c.layer[k];
    if (c.hparams) ends.layer[k] = {l.g, l.g_matrix, l.g_row, l.momentum, l.m_matrix, l.m_row, l.weight, l.w_matrix, l.w_row, l.rows, l.cols, l.scale, 0};
    else ends.layer[k] = {l.g, l.g_matrix, l.g_row, nullptr, 0, 0, l.out, l.out_matrix, l.out_row, l.rows, l.cols, l.scale, 0};
  }
  Args a = {};
  int blocks;
  bool small = true;
  for (int k = 0; k < c.n_layers; ++k) small = small && place_of(c.layer[k].rows, c.layer[k].cols).mb <= kSmall;
  small = small && c.gain[c.steps] <= kSmallGain;
  if (small) {
    Coefs coefs;
    coefs.steps = c.steps;
    coefs.eps = c.eps;
    for (int k = 0; k < POP_NS_MAX_STEPS; ++k)
      for (int i = 0; i < 3; ++i) coefs.coef[k][i] = c.coef[k][i];
    blocks = lay_out(c, a, 0, [](const NsLayer& l, const Place&) { return pieces(l.rows > l.cols ? l.rows : l.cols); });
    k_gram64<G><<<dim3(blocks), kThreads, 0, stream>>>(a, ends, ws);
    blocks = lay_out(c, a, 0, [](const NsLayer&, const Place&) { return 1; });
    k_square64<<<dim3(blocks), kSquareThreads, 0, stream>>>(a, ends, coefs, ws);
    blocks = lay_out(c, a, 0, [](const NsLayer& l, const Place&) { return ((l.rows > l.cols ? l.rows : l.cols) + kChunk - 1) / kChunk; });
    k_last64<G><<<dim3(blocks), kThreads, 0, stream>>>(a, ends, ws);
    return hipGetLastError();
  }
  Bounds bounds;
  bounds.steps = c.steps;
  bounds.segment = c.segment;
  bounds.most = c.most;
  for (int k = 0; k < POP_NS_MAX_STEPS; ++k) {
    for (int i = 0; i < 3; ++i) bounds.coef[k][i] = c.coef[k][i];
    bounds.gain[k] = c.gain[k];
    bounds.q_most[k] = c.q_most[k];
  }
  bounds.gain[POP_NS_MAX_STEPS] = c.gain[POP_NS_MAX_STEPS];
  blocks = lay_out(c, a, 0, [](const NsLayer& l, const Place&) { return parts(l.rows, l.cols); });
  k_norms<G><<<dim3(blocks), kThreads, 0, stream>>>(a, ends, ws);
  if (c.steps == 0) {
    k_no_steps<G><<<dim3(blocks), kThreads, 0, stream>>>(a, ends, ws);
    return hipGetLastError();
  }
  blocks = lay_out(c, a, 0, [](const NsLayer&, const Place& p) { return (p.mb * p.nb + 3) / 4; });
  k_start<G><<<dim3(blocks), kThreads, 0, stream>>>(a, bounds, ends, ws);
  const NoEnds none;
  const auto square = [](const Place&, int m, int) { return tiles(m); };
  const auto full = [](const Place&, int m, int n) { return m * n; };
  for (int first = 0, xt = 0; first < c.steps; first += c.segment, xt ^= 1) {
    const int last = (first + c.segment < c.steps ? first + c.segment : c.steps) - 1;
    launch_product<kGram, float>(c, args_of(first, first, last, xt), none, ws, stream, square);
    for (int k = first; k <= last; ++k) {
      const Args s = args_of(k, first, last, xt);
      launch_product<kPoly, float>(c, s, none, ws, stream, square);
      launch_product<kMix, float>(c, s, none, ws, stream, [&](const Place& p, int m, int n) { return square(p, m, n) * ((k > first) + (k < last)); });
      if (k < last) launch_product<kNext, float>(c, s, none, ws, stream, square);
    }
    const Args s = args_of(last, first, last, xt);
    if (last + 1 < c.steps) launch_product<kApply, float>(c, s, none, ws, stream, full);
    else launch_product<kLast, G>(c, s, ends, ws, stream, full);
  }
  return hipGetLastError();
}

}  // namespace ns
}  // namespace

// k_norms; k_start; k_tile of 128 x 128, two of whose products may share a launch; k_square64 (of 512 work items) and k_last64.  The
// other tilings are those of launches of few tiles (launch_product).
int64_t ns_most_workgroups(int64_t rows, int64_t cols) {
  const ns::Place p = ns::place_of((int)rows, (int)cols);
  const int64_t mt = (p.mb + ns::kTile - 1) / ns::kTile, nt = (p.nb + ns::kTile - 1) / ns::kTile, n = rows < cols ? cols : rows;
  int64_t most = ns::parts((int)rows, (int)cols);
  for (const int64_t w : {(int64_t)p.mb * p.nb / 4 + 1, mt * (mt + 1), mt * nt, p.mb <= ns::kSmall ? (n + ns::kChunk - 1) / ns::kChunk : 0})
    if (w > most) most = w;
  return most;
}

int64_t ns_workspace_bytes(int count, int rows, int cols) {
  const ns::Place p = ns::place_of(rows, cols);
  const int side = ns::small_side(rows < cols ? rows : cols);
  const int64_t small = p.mb <= ns::kSmall ? (int64_t)(ns::pieces(rows < cols ? cols : rows) + 1) * side * side * 8 : 0;
  return ns::head_bytes(count) + count * (p.size * 2 > small ? p.size * 2 : small);        // of whole 2 KB
}

hipError_t launch_ns(const NsCall& c, int dtype, void* ws, hipStream_t s) {
  return dtype == POP_F32 ? ns::run<float>(c, (char*)ws, s) : dtype == POP_BF16 ? ns::run<__bf16>(c, (char*)ws, s) : ns::run<_Float16>(c, (char*)ws, s);
}

}  // namespace pop
