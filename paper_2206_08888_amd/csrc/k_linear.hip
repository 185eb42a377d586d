// Linear attention with a decay for each head over sequences, its backward pass, and single steps (operators.h).
//
// Sequences go in chunks of 32 steps.  With S the state in front of a chunk and i, j its steps from 0 on,
//
//   o_i = read (lambda^(i+1) S^T q_i + write sum_{j <= i} lambda^(i-j) (k_j . q_i) v_j),    S' = lambda^32 S + write sum_j lambda^(31-j) k_j v_j^T
//
// and where episodes start, pairs of steps in different ones have weight 0 and the state reaches steps in front of the first start only.
// All sums are products of 16 x 16 x 32 on the bf16 matrix instructions, operands in exact or 24 bit parts (Parts), sums in fp32.  The
// three gradients are the same sums with other roles (op_api.hip): dq with d_o, v, k for q, k, v and the states turned over; dv and dk from
// the end with k, q, d_o and v, d_o, q.  They go in one launch.
//
// A workgroup has a column (agent, sequence, head) and walks its chunks: vectors of the next chunk are loaded while this one is computed,
// split into parts and laid into LDS, keys a second time times their weight in S'; three wavefronts compute the weights of pairs for
// all; each wavefront holds 16 columns of S in registers, as sums of the matrix instructions that are operands of the next ones as they are.
// Two barriers a chunk.
//
// What bounds it: at 64 x 64 in bf16 the issue of vector instructions, most of which split operands (80 x 8 x 512 x 4 heads: forward 179 us where
// the bytes alone take 139 at a large copy's rate, vector instructions issue in 73 % of a CU's busy cycles, LDS works in 43 %, matrix units in
// 23 %; three gradients 484 us, 237 at least, 80 / 49 / 26 %).  At 128 x 128 in fp16 nothing is busy half of the time (three gradients of 2 x 2 x 16383 x 4
// heads 488 us, 45 / 39 / 29 %): 85 KB of LDS are one workgroup on a CU, two wavefronts on a SIMD, which wait 40 % of their time, as a chunk is
// staged, a barrier, products, a barrier and outputs one after the other.  So are fp32 (six products for one, 63 KB of LDS for 64 x 64, two
// workgroups on a CU) and few columns, where a wavefront waits 35 to 40 %.  Chunks of 64 steps need the registers of two; 32 columns
// a wavefront, which would halve the reads of LDS, do not fit either.
#include <hip/hip_runtime.h>
#include <math.h>
#include <algorithm>
#include "operators.h"

namespace pop {
namespace {
namespace linear {

constexpr int kMost = POP_LINEAR_MAX_DIM;

__device__ inline float log_decay_of(const float* log_decay, int at) {
  const float z = log_decay ? log_decay[at] : 0.0f;
  return z > 0.0f ? 0.0f : z < -200.0f ? -200.0f : z;
}
template <typename E> __device__ inline const E* at(const pop_heads& s, int p, int b, int h) { return (const E*)s.data + p * s.agent + b * s.row + h * s.head; }

// ---- sequences

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
#define POP_LDS __attribute__((address_space(3)))

// Operands of a product are sums of bf16 parts: an array's values exactly (kIn of them); a computed operand (a weight, a state, keys times
// their decay) to 24 bits, as fp32 has it, whatever the arrays' type: states are fp32, and where sums cancel what is cut off in front of
// the output's rounding is all that is left.  (Two parts, 16 bits, for 16-bit arrays: forward and backward of 80 x 8 x 512 x 4 heads of 64 in
// bf16 587 us instead of 655, of 2 x 2 x 16383 x 4 heads of 128 in fp16 760 instead of 790.)
// Where both operands are arrays' values, products take them as they are where there are instructions for the type: kRaw parts.
constexpr int kOf = 3;
template <typename E> struct Parts { static constexpr int kIn = 2, kRaw = 1; };
template <> struct Parts<__bf16> { static constexpr int kIn = 1, kRaw = 1; };
template <> struct Parts<float> { static constexpr int kIn = 3, kRaw = 3; };

// An operand of v_mfma_f32_16x16x32_bf16: lane l has row (or column) l % 16 and the 8 places 4 g + j and 16 + 4 g + j, j = 0 .. 3, g = l / 16,
// of the 32 that are summed over.  Their order is free as long as both operands have the same, and in this one two results one under the
// other (rows 4 g + j of each) are an operand as they are.
template <int N> struct Operand { u32x4 part[N]; };

__device__ inline unsigned upper_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ inline float cut_off(float a) { return __uint_as_float(__float_as_uint(a) & 0xffff0000u); }
__device__ inline unsigned rounded(float a, float b) {
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  const pair p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(unsigned, p);
}
// Part after part is cut off and subtracted, the last one rounded.
template <int N> __device__ inline void split(float a, float b, unsigned (&part)[N]) {
#pragma unroll
  for (int n = 0; n + 1 < N; ++n) {
    part[n] = upper_halves(a, b);
    a -= cut_off(a);
    b -= cut_off(b);
  }
  part[N - 1] = rounded(a, b);
}
template <int N> __device__ inline Operand<N> operand(const f32x4& lo, const f32x4& hi) {
  Operand<N> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned part[N];
    split<N>(i < 2 ? lo[2 * i] : hi[2 * i - 4], i < 2 ? lo[2 * i + 1] : hi[2 * i - 3], part);
#pragma unroll
    for (int n = 0; n < N; ++n) o.part[n][i] = part[n];
  }
  return o;
}
// c + a b.  Parts that were cut off are below 2^-7 and 2^-15 of the value; of their products the ones below 2^-22 are left out: 2^-24 of a b on
// the average, as much as a product in fp32 is rounded by, and 2^-21 at most (nothing where one operand is a single part).
template <int A, int B> __device__ inline f32x4 product(const Operand<A>& a, const Operand<B>& b, f32x4 c) {
  constexpr int N = A > B ? A : B;
#pragma unroll
  for (int n = N - 1; n >= 0; --n)
#pragma unroll
    for (int i = 0; i < A; ++i)
      if (n - i >= 0 && n - i < B)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.part[i]), __builtin_bit_cast(bf16x8, b.part[n - i]), c, 0, 0, 0);
  return c;
}

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
template <typename E, int N> __device__ inline f32x4 product_of_values(const Operand<N>& a, const Operand<N>& b, f32x4 c) {
  if constexpr (__is_same(E, _Float16)) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.part[0]), __builtin_bit_cast(f16x8, b.part[0]), c, 0, 0, 0);
  else return product(a, b, c);
}

__device__ inline void sync_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// How a call's sequences are shared: `segments` of `per` chunks each, which go from the states that k_scan leaves.
struct Share { int chunks, per, segments, jobs; };
enum { kMain = 0, kStates = 1 };

// What Tile::below compares with for values that are finite and of magnitudes below 2^e: bits of 2^e without the sign for fp32; for two
// 16-bit values, what brings an exponent from e on to the sign's place.
constexpr int kFinite = 128;
template <typename E> __host__ __device__ constexpr unsigned border_of(int e) {
  constexpr bool half = __is_same(E, _Float16);
  const int exponent = e + (half ? 15 : 127), most = half ? 31 : 255;
  const unsigned first = (unsigned)(exponent < most ? exponent : most);
  return sizeof(E) == 4 ? first << 24 : (0x8000u - (first << (half ? 10 : 7))) * 0x10001u;
}

// How a call's arrays are reached.  kWide: vectors of 16 bytes from where they are aligned and a row has whole ones, four columns of o at a
// time; kNarrow: vectors that are aligned to elements only, the last one of a row moved back to where it ends with it (rows of less than
// a vector by elements); kAny: elements by addresses of 64 bits, for steps further apart than 32 bits reach, and steps that lie over
// each other.
enum { kWide = 0, kNarrow = 1, kAny = 2 };

// One array of a workgroup's sequence and head, a chunk of C steps after the other (in reverse one before the other): a buffer resource
// of the chunk's first `n` steps, behind whose end loads give zero and stores do nothing.
template <typename E, int C, int HOW> struct Steps {
  typedef __amdgpu_buffer_rsrc_t Rsrc;
  E* now;
  int64_t step, hop;
  int width, bytes;
  __device__ inline Steps(const pop_heads& s, int p, int b, int h, int width, int t, bool reverse)
      : now((E*)linear::at<E>(s, p, b, h) + t * s.step), step(s.step), hop(reverse ? -C * s.step : C * s.step), width(width) {
    bytes = (int)(((C - 1) * step + width) * (int64_t)sizeof(E));
  }
  __device__ inline Rsrc chunk(int n) const {
    return __builtin_amdgcn_make_buffer_rsrc(now, 0, n == C ? bytes : ((n - 1) * (int)step + width) * (int)sizeof(E), 0x00020000);
  }
  // The offset of element `c` of the chunk's step m in bytes.
  __device__ inline int offset(int m, int c) const { return c < width ? (m * (int)step + c) * (int)sizeof(E) : 0x70000000; }
  __device__ inline E element(Rsrc r, int n, int m, int c) const {
    if constexpr (HOW == kAny) return m < n && c < width ? now[m * step + c] : (E)0.0f;
    else if constexpr (sizeof(E) == 4) return __builtin_bit_cast(E, __builtin_amdgcn_raw_buffer_load_b32(r, offset(m, c), 0, 0));
    else return __builtin_bit_cast(E, __builtin_amdgcn_raw_buffer_load_b16(r, offset(m, c), 0, 0));
  }
  __device__ inline void put(Rsrc r, int n, int m, int c, E v) const {
    if constexpr (HOW == kAny) { if (m < n && c < width) now[m * step + c] = v; }
    else if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), r, offset(m, c), 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, v), r, offset(m, c), 0, 0);
  }
};

// What follows from the value is computed where it is used, not kept in registers through the loop: for paths that few calls take.
__device__ inline int here_only(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// The channel that row 4 g + i of tile d of the state stands for.
__device__ inline int channel_of(int d, int g, int i) { return 16 * d + 4 * g + i; }

// C steps of an array's channels: the threads of the workgroup take vectors of 16 bytes in turn.  Row r of a chunk is its step r, from the
// end in reverse.
template <typename E, int KB, int NW, int C, int HOW> struct Tile {
  static constexpr int kVec = 16 / sizeof(E), kAcross = 32 * KB / kVec, kAll = C * kAcross, kEach = (kAll + 64 * NW - 1) / (64 * NW);
  // Planes that rows are read of and ones that are turned over: strides that spread a read's lanes over all banks (all planes with the first
  // stride, forward and backward of 2 x 2 x 16383 x 4 heads of 128, fp16: 816 against 787 us).
  static constexpr int kStride = 32 * KB + 8, kPlane = C * kStride, kTurned = 32 * KB + 16, kTurnedPlane = C * kTurned, kIn = Parts<E>::kIn, kRaw = Parts<E>::kRaw, kPairs = kVec / 2;
  typedef unsigned Word __attribute__((ext_vector_type(kPairs)));    // a vector's values, one part of each
  u32x4 v[kEach];
  static __device__ inline bool whole(int i) { return kAll % (64 * NW) == 0 || row(i) < C; }
  static __device__ inline int row(int i, int thread = threadIdx.x) { return (thread + i * 64 * NW) / kAcross; }
  // The step of the chunk that a vector is of: not in front of the array for threads behind the last row either.
  static __device__ inline int step(int i, bool reverse, int thread) {
    const int m = reverse ? C - 1 - row(i, thread) : row(i, thread);
    return kAll % (64 * NW) == 0 ? m : max(m, 0);
  }
  static __device__ inline int channel(int i, int thread = threadIdx.x) { return (thread + i * 64 * NW) % kAcross * kVec; }
  static __device__ inline int thread() { return HOW == kWide ? (int)threadIdx.x : here_only(threadIdx.x); }
  __device__ inline void load(const Steps<E, C, HOW>& a, int n, bool reverse) {
    const auto r = a.chunk(n);
    const int id = thread();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int m = step(i, reverse, id);
      if constexpr (HOW == kWide) {
        v[i] = __builtin_amdgcn_raw_buffer_load_b128(r, a.offset(m, channel(i, id)), 0, 0);
      } else {
        if (HOW == kNarrow && a.width >= kVec) {                     // in front of the end of an existing row, whatever is asked for
          const unsigned at = (unsigned)(min(m, n - 1) * (int)a.step + min(channel(i, id), a.width - kVec));
          __builtin_memcpy(&v[i], a.now + at, 16);
        } else {
          E e[kVec];
#pragma unroll
          for (int k = 0; k < kVec; ++k) e[k] = a.element(r, n, m, channel(i, id) + k);
          __builtin_memcpy(&v[i], e, 16);
        }
      }
    }
  }
  // What was asked for: values of the vector moved to their places, zeros behind the ends of rows and behind the last one.
  __device__ inline void settle(const Steps<E, C, HOW>& a, int n, bool reverse) {
    if (HOW != kNarrow || a.width < kVec) return;
    const int id = thread();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int m = step(i, reverse, id), off = max(0, channel(i, id) - (a.width - kVec)) * (int)sizeof(E) * 8;
      uint64_t lo = v[i][0] | (uint64_t)v[i][1] << 32, hi = v[i][2] | (uint64_t)v[i][3] << 32;
      if (off >= 64) {
        lo = hi;
        hi = 0;
      }
      const int by = off & 63;
      lo = lo >> by | hi << 1 << (63 - by);
      hi >>= by;
      const bool none = m >= n || off >= 128;
      v[i] = u32x4{none ? 0 : (unsigned)lo, none ? 0 : (unsigned)(lo >> 32), none ? 0 : (unsigned)hi, none ? 0 : (unsigned)(hi >> 32)};
    }
  }
  // Whether all values are finite and below a border (border_of).
  __device__ inline bool below(unsigned border) const {
    unsigned bad = 0, most = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (!whole(i)) break;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const unsigned w = v[i][d];
        if constexpr (sizeof(E) == 4) most = max(most, w << 1);
        else bad |= (w & (__is_same(E, _Float16) ? 0x7c007c00u : 0x7f807f80u)) + border;
      }
    }
    return sizeof(E) == 4 ? most < border : (bad & 0x80008000u) == 0;
  }
  __device__ inline void pair(int i, int d, float& a, float& b) const {
    if constexpr (sizeof(E) == 4) {
      a = __uint_as_float(v[i][2 * d]);
      b = __uint_as_float(v[i][2 * d + 1]);
    } else {
      typedef E Two __attribute__((ext_vector_type(2)));
      const unsigned w = v[i][d];                                    // (of an element in its place the cast takes the first)
      const Two x = __builtin_bit_cast(Two, w);
      a = (float)x[0];
      b = (float)x[1];
    }
  }
  template <bool TURNED> static __device__ inline unsigned short* place(unsigned short* plane, int i) { return plane + row(i) * (TURNED ? kTurned : kStride) + channel(i); }
  // Into LDS, part by part, or as they are.
  template <int N, bool TURNED> __device__ inline void store(unsigned short* plane) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (!whole(i)) break;
      if constexpr (N == 1) *(u32x4*)place<TURNED>(plane, i) = v[i];
      else put<N, TURNED>(plane, i, 1.0f, false);
    }
  }
  // Vector i times f.
  template <int N, bool TURNED> __device__ inline void put(unsigned short* plane, int i, float f, bool times) const {
    Word word[N];
#pragma unroll
    for (int d = 0; d < kPairs; ++d) {
      float a, b;
      pair(i, d, a, b);
      unsigned part[N];
      if (times) split<N>(a * f, b * f, part);
      else split<N>(a, b, part);
#pragma unroll
      for (int n = 0; n < N; ++n) word[n][d] = part[n];
    }
#pragma unroll
    for (int n = 0; n < N; ++n) *(Word*)(place<TURNED>(plane, i) + n * (TURNED ? kTurnedPlane : kPlane)) = word[n];
  }
  // Rows 16 tile .. of 32 channels as an operand: a lane has channels 8 g .. 8 g + 7.
  template <int N> static __device__ inline Operand<N> rows(const unsigned short* plane, int tile, int kb, int lane) {
    Operand<N> o;
    const unsigned short* from = plane + (16 * tile + (lane & 15)) * kStride + 32 * kb + 8 * (lane >> 4);
#pragma unroll
    for (int n = 0; n < N; ++n) o.part[n] = *(const u32x4*)(from + n * kPlane);
    return o;
  }
  // The same, a lane with channels 4 g .. 4 g + 3 and 16 + 4 g .. as two tiles of the state have them.
  template <int N> static __device__ inline Operand<N> rows_in_tiles(const unsigned short* plane, int tile, int kb, int lane) {
    Operand<N> o;
    const unsigned short* from = plane + (16 * tile + (lane & 15)) * kStride + 32 * kb + 4 * (lane >> 4);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const u32x2 x = *(const u32x2*)(from + n * kPlane), y = *(const u32x2*)(from + n * kPlane + 16);
      o.part[n] = u32x4{x[0], x[1], y[0], y[1]};
    }
    return o;
  }
  // Channels 16 d .. 16 d + 15 of 32 rows as an operand, four rows of four times four channels turned over by the read.
  template <int N> static __device__ inline Operand<N> channels(unsigned short* plane, int d, int lane) {
    Operand<N> o;
    unsigned short* from = plane + (4 * (lane >> 4) + (lane & 15) / 4) * kTurned + channel_of(d, lane & 3, 0);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((POP_LDS s16x4*)(from + n * kTurnedPlane));
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((POP_LDS s16x4*)(from + n * kTurnedPlane + 16 * kTurned));
      const u32x2 x = __builtin_bit_cast(u32x2, a), y = __builtin_bit_cast(u32x2, b);
      o.part[n] = u32x4{x[0], x[1], y[0], y[1]};
    }
    return o;
  }
};

__device__ inline float power(float log2_decay, int n) { return __builtin_amdgcn_exp2f((float)n * log2_decay); }
__device__ inline bool not_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }
__device__ inline bool any_lane(bool v) { return __builtin_amdgcn_ballot_w64(v) != 0; }

// A chunk without starts of episodes and with all of its steps is computed apart, without what the others check (forward and backward of 2 x 2 x
// 16383 x 4 heads of 128, fp16: 805 -> 787 us; of 80 x 8 x 512 x 4 heads of 64, bf16: 655 -> 650).
template <bool YES> struct Plain { static constexpr bool yes = YES; };

constexpr int kGroups = 1 << 15;       // of 8 columns, in x of a grid: its work items stay below 2^32

// What registers allow without spills (the build refuses kernels that spill).
template <typename E, int KB> constexpr int waves_per_simd() { return KB > 2 ? 2 : sizeof(E) == 4 ? (KB == 1 ? 3 : 2) : __is_same(E, __bf16) || KB == 1 ? 4 : 3; }

// A wavefront has 16 of the state's columns, the workgroup those of NW wavefronts.
template <typename E, int KB, int NW, int C, int HOW>
__global__ void __launch_bounds__(64 * NW, (waves_per_simd<E, KB>())) k_chunks(LinearArgs a, Share share, float* ws, int mode, int jobs) {
  typedef Tile<E, KB, NW, C, HOW> T;
  typedef Tile<E, NW / 2, NW, C, HOW> TV;
  typedef Steps<E, C, HOW> Array;
  constexpr int kIn = Parts<E>::kIn, kRaw = Parts<E>::kRaw;
  constexpr bool kTwice = kIn != kRaw;                               // queries in parts and as they are
  static_assert(C == 32, "two tiles of rows; starts of episodes are the bits of a word");
  __shared__ __attribute__((aligned(16))) unsigned short keys[kRaw * T::kPlane], queries[kIn * T::kPlane], asked[kTwice ? kRaw * T::kPlane : 8], faded[kOf * T::kTurnedPlane], values[kIn * TV::kTurnedPlane];
  __shared__ u32x2 shared_weights[3][kOf][64];
  __shared__ int bad[2];
  // the roles of a column one after the other on one XCD: they read the same arrays
  const int job = blockIdx.x / 8 % jobs, unit = (blockIdx.y * kGroups + blockIdx.x / (8 * jobs)) * 8 + blockIdx.x % 8, cols = a.P * a.B * a.H;
  if (unit >= cols * share.segments) return;
  const LinearRole& role = a.role[job];
  const int seg = unit / cols, col = unit - seg * cols, h = col % a.H, row = col / a.H, b = row % a.B, p = row / a.B;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, at = lane & 15, K = role.K, V = role.V;
  const bool reverse = role.reverse, states = mode == kStates;
  const int len = a.lengths ? min(max(a.lengths[row], 0), a.T) : a.T;
  const uint8_t* reset = a.reset.data ? (const uint8_t*)a.reset.data + p * a.reset.agent + b * a.reset.row : nullptr;
  const float l2 = log_decay_of(a.log_decay, p * a.H + h) * 1.44269504f, lambda = power(l2, 1);
  const int behind = reverse ? 1 : 0;                               // factors of the state on its way out, beside those between rows (on its way in: 1 - behind)
  const int segment = reverse ? share.segments - 1 - seg : seg, from = min(segment * share.per, share.chunks), until = min(from + share.per, share.chunks);
  const int start = from * C, end = min(until * C, a.T), n_chunks = max(0, (min(end, len) - start + C - 1) / C);
  const int first_t = start + (reverse ? max(n_chunks - 1, 0) * C : 0);
  Array q(role.q, p, b, h, K, first_t, reverse), k(role.k, p, b, h, K, first_t, reverse), v(role.v, p, b, h, V, first_t, reverse), o(role.o, p, b, h, V, first_t, reverse);
  const bool idle = 16 * wave >= V;                                  // a wave with no columns loads with the others

  // the state: S[d][i] is channel channel_of(d, g, i) of this lane's column
  f32x4 S[2 * KB];
  bool tainted = false;
  {
    const float* first = states ? nullptr : share.segments > 1 ? ws : role.first;
    int64_t base = (int64_t)col * K * V;
    int along_k = role.first_k, along_v = role.first_v;
    if (share.segments > 1) {
      // role 2 takes the states of role 1, transposed
      base += ((int64_t)min(job, 1) * share.segments + seg) * cols * K * V;
      along_k = job == 2 ? 1 : V;
      along_v = job == 2 ? K : 1;
    }
    const int g = here_only(lane) >> 4, column = 16 * wave + (here_only(lane) & 15);
#pragma unroll
    for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row_k = channel_of(d, g, i);
        S[d][i] = first && row_k < K && column < V ? first[base + row_k * along_k + column * along_v] : 0.0f;
        tainted |= not_finite(S[d][i]);
      }
    tainted = any_lane(tainted);
  }

  // Weights of this thread's rows of keys on their way out.
  const float both = role.read * role.write, whole = power(l2, C);
  float outof[T::kEach];
#pragma unroll
  for (int i = 0; i < T::kEach; ++i) outof[i] = role.write * power(l2, max(C - 1 - T::row(i), 0) + behind);

  T next_k, next_q;
  TV next_v;
  uint8_t next_cut = 0;
  const auto load = [&](int n) {
    const int t = start + (reverse ? n_chunks - 1 - n : n) * C, count = min(C, len - t);
    next_k.load(k, count, reverse);
    if (!states) next_q.load(q, count, reverse);
    next_v.load(v, count, reverse);
    k.now += k.hop;
    q.now += q.hop;
    v.now += v.hop;
    if (reset) {
      const int m = reverse ? C - lane : lane;                       // in reverse what leads from the step behind to row `lane`
      next_cut = lane < C && t + m < len && m < count + (reverse ? 1 : 0) ? reset[(int64_t)(t + m) * a.reset.step] : 0;
    }
  };
  if (n_chunks > 0) load(0);
  if (threadIdx.x == 0) bad[0] = 0;
  sync_lds();
  if (tainted) bad[0] = 1;
  bool any_cut = false;

  int n = 0;
  for (; n < n_chunks; ++n) {
    const int t = start + (reverse ? n_chunks - 1 - n : n) * C, count = min(C, len - t);
    if (n > 0) o.now += o.hop;
    const unsigned cuts = (unsigned)__builtin_amdgcn_ballot_w64(next_cut != 0);
    any_cut |= cuts != 0;
    const bool regular = cuts == 0 && count == C;
    const auto starts = [&](int r) { return __popc(cuts & ((2u << here_only(r)) - 1)); };   // episodes that start at rows 0 .. r
    const int all_starts = __popc(cuts);
    next_k.settle(k, count, reverse);
    next_v.settle(v, count, reverse);
    next_v.template store<kIn, true>(values);
    // fp16 values' products are below 2^39, and the boundary knows the scale: a constant (forward and backward of 2 x 2 x 16383 x 4 heads of
    // 128: 790 us, with the argument 812)
    const unsigned border = __is_same(E, _Float16) ? border_of<E>(kFinite) : a.border;
    bool fine = next_k.below(border) & next_v.below(border_of<E>(kFinite));
    if (!states) {
      next_q.settle(q, count, reverse);
      next_k.template store<kRaw, false>(keys);
      next_q.template store<kIn, false>(queries);
      if constexpr (kTwice) next_q.template store<kRaw, false>(asked);
      fine &= next_q.below(border);
    }
    if (!fine) bad[n & 1] = 1;
#pragma unroll
    for (int i = 0; i < T::kEach; ++i) {
      if (!T::whole(i)) break;
      float f = outof[i];
      if (!regular) {
        const int r = here_only(T::row(i));
        if (!reverse) f = role.write * power(l2, max(count - 1 - r, 0));
        f = starts(r) == all_starts ? f : 0.0f;
      }
      next_k.template put<kOf, true>(faded, i, f, true);
    }
    sync_lds();
    if (n + 1 < n_chunks) load(n + 1);
    const int not_fine = bad[n & 1];
    if (threadIdx.x == 0) bad[(n + 1) & 1] = 0;

    f32x4 out[2];                                                    // rows: columns 4 g + i of the wave's; column: row `at` of the tile
    Operand<kIn> value;
    const auto pairs = [&](auto plain) {
      // the weights of pairs of rows, for all wavefronts: tiles 0 and 1 with themselves, 1 with 0
      for (int w = NW - 1 - wave; w < 3; w += NW) {
        const int queried = w > 0, other = w == 1;
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int d = 0; d < KB; ++d) x = product_of_values<E>(T::template rows<kRaw>(keys, other, d, lane), T::template rows<kRaw>(kTwice ? asked : queries, queried, d, lane), x);
        // row `at` of the one and row 4 g + j of the other
        const int first = here_only(at - 4 * g) + (w < 2 ? 0 : 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = first >= j ? x[j] * (both * power(l2, first - j)) : 0.0f;
        if constexpr (!plain.yes) {
          const int mine = starts(16 * queried + at);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = starts(16 * other + 4 * g + j) == mine ? x[j] : 0.0f;
        }
        unsigned lo[kOf], hi[kOf];
        split<kOf>(x[0], x[1], lo);
        split<kOf>(x[2], x[3], hi);
#pragma unroll
        for (int n = 0; n < kOf; ++n) shared_weights[w][n][lane] = u32x2{lo[n], hi[n]};
      }
    };
    const auto from_state = [&](auto plain) {
      Operand<kOf> memory[KB];
#pragma unroll
      for (int d = 0; d < KB; ++d) memory[d] = operand<kOf>(S[2 * d], S[2 * d + 1]);
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) out[tile] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int d = 0; d < KB; ++d)
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) out[tile] = product(memory[d], T::template rows_in_tiles<kIn>(queries, tile, d, lane), out[tile]);
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) {
        const int i = 16 * tile + here_only(at);                     // (found again: a register that the bf16 kernels do not have)
        out[tile] *= role.read * power(l2, reverse ? max(i - (C - count), 0) : i + 1);
        if constexpr (!plain.yes) {
          const bool own = starts(16 * tile + at) != 0;              // nothing of the state
#pragma unroll
          for (int e = 0; e < 4; ++e) out[tile][e] = own ? 0.0f : out[tile][e];
        }
      }
    };
    const auto next_state = [&](auto plain) {
      if constexpr (!plain.yes) {
        const float keep = power(l2, count);
#pragma unroll
        for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) S[d][i] = all_starts == 0 ? S[d][i] * keep : 0.0f;
      } else {
#pragma unroll
        for (int d = 0; d < 2 * KB; ++d) S[d] *= whole;
      }
#pragma unroll
      for (int d = 0; d < 2 * KB; ++d) S[d] = product(T::template channels<kOf>(faded, d, lane), value, S[d]);
    };
    if (!states) {
      if (regular) pairs(Plain<true>());
      else pairs(Plain<false>());
      if (!idle) {
        if (regular) from_state(Plain<true>());
        else from_state(Plain<false>());
      }
    }
    // A product with a weight of zero would carry what is not finite where it does not belong, and products of keys and queries may be
    // beyond fp32's range where those with the state are not: the rest goes step by step.
    if (__builtin_amdgcn_readfirstlane(not_fine) != 0) break;
    if (!idle) {
      value = TV::template channels<kIn>(values, wave, lane);
      if (regular) next_state(Plain<true>());
      else next_state(Plain<false>());
    }
    sync_lds();                                                      // all of the chunk has been read but the weights, which are written

    if (states || idle) continue;
    const auto r = o.chunk(count);
    const int id = HOW == kWide ? lane : here_only(lane);
#pragma unroll
    for (int tile = 0; tile < 2; ++tile) {
      Operand<kOf> weights;
#pragma unroll
      for (int n = 0; n < kOf; ++n) {
        const u32x2 lo = shared_weights[tile == 0 ? 0 : 2][n][lane], hi = shared_weights[1][n][lane];
        weights.part[n] = tile == 0 ? u32x4{lo[0], lo[1], 0, 0} : u32x4{lo[0], lo[1], hi[0], hi[1]};
      }
      const f32x4 y = product(value, weights, out[tile]);
      typedef E Four __attribute__((ext_vector_type(4)));
      const Four x = {(E)y[0], (E)y[1], (E)y[2], (E)y[3]};
      const int i = 16 * tile + (id & 15), m = reverse ? C - 1 - i : i, column = 16 * wave + 4 * (id >> 4);
      if constexpr (HOW == kWide) {
        if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), r, o.offset(m, column), 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, x), r, o.offset(m, column), 0, 0);
      } else {
        if (HOW == kNarrow && column + 4 <= V) {
          if (m < count) __builtin_memcpy(o.now + (unsigned)(m * (int)o.step + column), &x, sizeof(Four));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const E y = x[e];
            o.put(r, count, m, column + e, y);
          }
        }
      }
    }
  }

  if (n < n_chunks && !idle) {
    const int first = start + (reverse ? 0 : n * C), behind = reverse ? start + min((n_chunks - n) * C, len - start) : min(end, len);
    const E *qs = linear::at<E>(role.q, p, b, h), *ks = linear::at<E>(role.k, p, b, h), *vs = linear::at<E>(role.v, p, b, h);
    E* os = (E*)linear::at<E>(role.o, p, b, h);
    const int g = here_only(lane) >> 4, column = 16 * wave + (here_only(lane) & 15);
#pragma unroll 1
    for (int i = first; i < behind; ++i) {
      const int64_t s = reverse ? first + behind - 1 - i : i;
      const bool cut = reset && (!reverse || s + 1 < len) && reset[(s + (reverse ? 1 : 0)) * a.reset.step];
      any_cut |= cut;
      const float vr = column < V ? (float)vs[s * role.v.step + column] : 0.0f;
      float sum = 0.0f;
#pragma unroll
      for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int kr = channel_of(d, g, i);
          if (kr < K) {
            // the smaller one of the two times a factor above 1, the larger one times one below: within the range where all three are (fp16
            // values times their scales always are)
            const float key = (float)ks[s * role.k.step + kr];
            const bool on_key = !__is_same(E, _Float16) && (fabsf(key) < fabsf(vr)) == (fabsf(role.write) > 1.0f);
            const float x = fmaf(on_key ? key * role.write : key, on_key ? vr : vr * role.write, cut ? 0.0f : reverse ? S[d][i] : lambda * S[d][i]);
            if (!states) sum = fmaf((float)qs[s * role.q.step + kr], x, sum);
            S[d][i] = reverse ? lambda * x : x;
          }
        }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (!states && g == 0 && column < V) os[s * role.o.step + column] = (E)(sum * role.read);
    }
  }

  const int behind_g = here_only(lane) >> 4, column = 16 * wave + (here_only(lane) & 15);
  if (!states && column < V)
    for (int t = max(start, len) + behind_g; t < end; t += 4) ((E*)linear::at<E>(role.o, p, b, h))[t * role.o.step + column] = (E)0.0f;
  const bool last = seg == share.segments - 1;
  float* to = states ? ws + (((int64_t)job * share.segments + seg) * cols + col) * K * V : last && role.last ? role.last + (int64_t)col * K * V : nullptr;
  if (!to) return;
  const bool cut = !states && reverse && len > 0 && reset && reset[0];
#pragma unroll
  for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row_k = channel_of(d, behind_g, i);
      if (row_k < K && column < V) to[row_k * V + column] = cut ? 0.0f : S[d][i];
    }
  if (states && threadIdx.x == 0) {
    float* factor = ws + (int64_t)share.jobs * share.segments * cols * K * V;
    factor[((int64_t)job * share.segments + seg) * cols + col] = any_cut ? -1.0f : power(l2, max(0, min(end, len) - start));
  }
}

// The states in front of the segments, in the places of what the segments add to them.  A negative factor: nothing of the state in front
// is left.  A workgroup has 64 elements of states, a wavefront AHEAD segments in a row: it finds what they do together, and with
// what those of the wavefronts in front do the states in front of each.  (192 segments of 4 states of 64 x 64, one after the other: 17 us.)
constexpr int kScan = 64;
template <int NW, int AHEAD> __global__ void __launch_bounds__(kScan * NW) k_scan(LinearArgs a, Share share, float* ws, int cols) {
  __shared__ float sums[NW][kScan], factors[NW][kScan];
  const LinearRole& role = a.role[blockIdx.y];
  const int size = role.K * role.V, n = cols * size, lane = threadIdx.x % kScan, wave = threadIdx.x / kScan;     // few columns: n is below 2^27
  const int i = min(blockIdx.x * kScan + lane, n - 1), col = i / size, e = i - col * size;
  const bool mine = blockIdx.x * kScan + lane < n;
  float* at = ws + (int64_t)blockIdx.y * share.segments * n + i;
  const float* factor = ws + (int64_t)share.jobs * share.segments * n + (int64_t)blockIdx.y * share.segments * cols + col;
  const auto behind = [](float s, float sum, float f) { return f < 0.0f ? sum : fmaf(f, s, sum); };
  float s = role.first ? role.first[(int64_t)col * size + e / role.V * role.first_k + e % role.V * role.first_v] : 0.0f;
  for (int all = 0; all < share.segments; all += NW * AHEAD) {
    const int k = all + wave * AHEAD;
    float add[AHEAD], f[AHEAD], sum = 0.0f, product = 1.0f;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int from = min(k + u, share.segments - 1);
      add[u] = at[(int64_t)from * n];
      f[u] = factor[from * cols];
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (k + u >= share.segments) continue;
      sum = behind(sum, add[u], f[u]);
      product = f[u] < 0.0f || product < 0.0f ? -1.0f : product * f[u];
    }
    if (NW > 1) {
      sums[wave][lane] = sum;
      factors[wave][lane] = product;
      __syncthreads();
      float in_front = s;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        if (w == wave) in_front = s;
        s = behind(s, sums[w][lane], factors[w][lane]);
      }
      if (all + NW * AHEAD < share.segments) __syncthreads();
      sum = in_front;
    } else {
      const float in_front = s;
      s = behind(s, sum, product);
      sum = in_front;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (k + u >= share.segments) continue;
      if (mine) at[(int64_t)(k + u) * n] = sum;
      sum = behind(sum, add[u], f[u]);
    }
  }
}

// Bound by reading and writing the states: 80 agents x 64 rows x 4 heads of 64 x 64, 546 MB, 104 us (5.2 TB/s; elements one by one: 146 us).
// A workgroup of NW wavefronts per row and head; a thread has four columns of every so many'th row of the state.
template <typename E, int NW> __global__ void __launch_bounds__(64 * NW) k_step(LinearStep a) {
  constexpr int kStep = 64 * NW, kRows = 4;
  __shared__ float sq[kMost], sk[kMost], part[NW][kMost];
  const int h = blockIdx.x % a.H, row = blockIdx.x / a.H, b = row % a.B, p = row / a.B;
  const int slot = a.slots ? a.slots[row] : b;
  E* o = (E*)a.o.data + p * a.o.agent + b * a.o.row + h * a.o.head;
  if (slot < 0 || slot >= a.n_slots) {
    for (int i = threadIdx.x; i < a.V; i += kStep) o[i] = (E)0.0f;
    return;
  }
  for (int i = threadIdx.x; i < a.K; i += kStep) {
    sq[i] = (float)at<E>(a.q, p, b, h)[i];
    sk[i] = (float)at<E>(a.k, p, b, h)[i];
  }
  const bool cut = a.reset.data && ((const uint8_t*)a.reset.data)[p * a.reset.agent + b * a.reset.row];
  const float lambda = expf(log_decay_of(a.log_decay, p * a.H + h));
  const int quads = (a.V + 3) / 4, shift = quads > 1 ? 32 - __clz(quads - 1) : 0, width = 1 << shift, hop = kStep >> shift;
  const int column = 4 * (threadIdx.x & (width - 1)), n = min(4, a.V - column);      // n <= 0: none
  float* S = a.state + (((int64_t)p * a.n_slots + slot) * a.H + h) * a.K * a.V + column;
  float v[4], sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = c < n ? (float)at<E>(a.v, p, b, h)[column + c] : 0.0f;
  for (int first = threadIdx.x >> shift; first - (int)(threadIdx.x >> shift) < a.K; first += kRows * hop) {
    f32x4 s[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int k = first + r * hop;
      s[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (!cut && k < a.K) {
        if (n == 4) __builtin_memcpy(&s[r], S + k * a.V, 16);
        else
#pragma unroll
          for (int c = 0; c < 3; ++c)
            if (c < n) s[r][c] = S[k * a.V + c];
      }
    }
    if (first == (int)(threadIdx.x >> shift)) __syncthreads();       // (for all threads in the first round)
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int k = first + r * hop;
      if (k < a.K) {
        const float key = sk[k], query = sq[k];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[r][c] = fmaf(key, v[c], lambda * s[r][c]);
          sum[c] = fmaf(query, s[r][c], sum[c]);
        }
        if (n == 4) __builtin_memcpy(S + k * a.V, &s[r], 16);
        else
#pragma unroll
          for (int c = 0; c < 3; ++c)
            if (c < n) S[k * a.V + c] = s[r][c];
      }
    }
  }
  for (int d = width; d < 64; d *= 2)
#pragma unroll
    for (int c = 0; c < 4; ++c) sum[c] += __shfl_xor(sum[c], d);
  if ((threadIdx.x & 63) < width)
#pragma unroll
    for (int c = 0; c < 4; ++c) part[threadIdx.x >> 6][column + c] = sum[c];
  __syncthreads();
  for (int i = threadIdx.x; i < a.V; i += kStep) {
    float all = part[0][i];
#pragma unroll
    for (int w = 1; w < NW; ++w) all += part[w][i];
    o[i] = (E)(all * a.scale);
  }
}

constexpr int kChunk = 32, kLeast = 4, kMostSegments = 4096, kCUs = 256, kLds = 160 << 10;
int blocks_of(int K) { return K <= 32 ? 1 : K <= 64 ? 2 : 4; }
int waves_of(int V) { return V <= 32 ? 2 : V <= 64 ? 4 : 8; }

// Workgroups that the card holds at once.
template <typename E, int KB> int64_t at_once(int waves) {
  typedef Parts<E> P;
  const int plane = 2 * kChunk * (32 * KB + 8), turned = 2 * kChunk * (32 * KB + 16), values = 2 * kChunk * (16 * waves + 16);
  const int lds = (P::kRaw + P::kIn + (P::kIn != P::kRaw ? P::kRaw : 0)) * plane + kOf * turned + P::kIn * values + 3 * kOf * 64 * 8 + 64;
  const int by_lds = kLds / lds, by_waves = 4 * waves_per_simd<E, KB>() / waves;
  return (int64_t)kCUs * (by_lds < by_waves ? by_lds : by_waves);
}
template <typename E> int64_t at_once(int K, int V) {
  const int kb = blocks_of(K), waves = waves_of(V);
  return kb == 1 ? at_once<E, 1>(waves) : kb == 2 ? at_once<E, 2>(waves) : at_once<E, 4>(waves);
}

// Sequences are cut into segments where there are too few of them, the segments' own states first, then those in front of them.  Roles go
// together, in a kernel that is wide enough for all.  Of the numbers of segments that fill whole rounds of workgroups, the one whose
// chunks one after the other take least: a chunk of states takes about half as long as one with outputs (28 / 50 us for 10 x 4 x 1000 x 4
// heads of 64, fp32), a workgroup's beginning and end as long as two chunks, the two launches more as long as two with outputs, the scan
// a fortieth of one for each segment.
Share share_of(int64_t cols, int64_t T, int K, int V, int dtype, bool backward) {
  const int64_t chunks = (T + kChunk - 1) / kChunk, roles = backward ? 3 : 1, jobs = backward ? 2 : 1;
  if (backward) K = V = K > V ? K : V;
  const int64_t slots = dtype == POP_F32 ? at_once<float>(K, V) : dtype == POP_BF16 ? at_once<__bf16>(K, V) : at_once<_Float16>(K, V);
  const auto rounds = [&](int64_t workgroups) { return (workgroups + slots - 1) / slots; };
  Share best = {(int)chunks, (int)chunks, 1, 0};
  int64_t least = 40 * (chunks + 2) * rounds(cols * roles);
  for (int n = 1; n <= 8; ++n)
    for (int64_t each : {cols * roles, cols * jobs}) {
      int64_t want = n * slots / each;
      if (want > kMostSegments) want = kMostSegments;
      if (want > chunks / kLeast) want = chunks / kLeast;
      if (want <= 1) continue;
      const int64_t per = (chunks + want - 1) / want, segments = (chunks + per - 1) / per;
      const int64_t cost = (per + 2) * (40 * rounds(cols * roles * segments) + 20 * rounds(cols * jobs * segments)) + 80 + segments;
      if (cost >= least) continue;
      least = cost;
      best = {(int)chunks, (int)per, (int)segments, (int)jobs};
    }
  return best;
}

typedef void (*Kernel)(LinearArgs, Share, float*, int, int);
template <typename E, int KB, int HOW> Kernel kernel_of(int V) {
  return waves_of(V) == 8 ? k_chunks<E, KB, 8, kChunk, HOW> : waves_of(V) == 4 ? k_chunks<E, KB, 4, kChunk, HOW> : k_chunks<E, KB, 2, kChunk, HOW>;
}
template <typename E, int HOW> Kernel kernel_of(int K, int V) {
  return blocks_of(K) == 1 ? kernel_of<E, 1, HOW>(V) : blocks_of(K) == 2 ? kernel_of<E, 2, HOW>(V) : kernel_of<E, 4, HOW>(V);
}
template <typename E> void launch(int how, const LinearArgs& a, const Share& share, float* ws, int mode, int jobs, int K, int V, hipStream_t s) {
  if (how == kAny) K = V = POP_LINEAR_MAX_DIM;
  const Kernel k = how == kWide ? kernel_of<E, kWide>(K, V) : how == kNarrow ? kernel_of<E, kNarrow>(K, V) : k_chunks<E, POP_LINEAR_MAX_DIM / 32, 8, kChunk, kAny>;
  const unsigned groups = (unsigned)((a.P * a.B * a.H * share.segments + 7) / 8), across = groups < kGroups ? groups : kGroups;
  k<<<dim3(across * 8 * jobs, (groups + across - 1) / across), 64 * waves_of(V), 0, s>>>(a, share, ws, mode, jobs);
}
template <typename E> int how_of(const LinearArgs& a) {
  int how = kWide;
  for (int i = 0; i < a.roles; ++i) {
    const LinearRole& r = a.role[i];
    const auto aligned = [](const pop_heads& s, int width, int n) {
      return width % n == 0 && (uintptr_t)s.data % (n * sizeof(E)) == 0 && s.agent % n == 0 && s.row % n == 0 && s.step % n == 0 && s.head % n == 0;
    };
    const auto near = [](const pop_heads& s, int width) { return s.step >= width && s.step < (int64_t)((1u << 30) / sizeof(E)) / kChunk; };
    if (!near(r.q, r.K) || !near(r.k, r.K) || !near(r.v, r.V) || !near(r.o, r.V)) return kAny;
    constexpr int n = 16 / sizeof(E);
    if (!aligned(r.q, r.K, n) || !aligned(r.k, r.K, n) || !aligned(r.v, r.V, n) || !aligned(r.o, r.V, 4)) how = kNarrow;
  }
  return how;
}
template <typename E> hipError_t run(LinearArgs a, int dtype, float* ws, hipStream_t s) {
  // read k . q write is below 2^(7 + 2 e) |read write| for 2^7 channels of magnitudes below 2^e: at most 2^127
  a.border = border_of<E>((120 - std::max(0, ilogbf(a.role[0].read * a.role[0].write) + 1)) / 2);
  const int cols = a.P * a.B * a.H;
  const Share share = share_of(cols, a.T, a.role[0].K, a.role[0].V, dtype, a.roles > 1);
  const int most = a.role[0].K > a.role[0].V ? a.role[0].K : a.role[0].V, K = a.roles > 1 ? most : a.role[0].K, V = a.roles > 1 ? most : a.role[0].V;
  const int how = how_of<E>(a);
  if (share.segments > 1) {
    launch<E>(how, a, share, ws, kStates, share.jobs, K, V, s);
    const dim3 grid((cols * a.role[0].K * a.role[0].V + kScan - 1) / kScan, share.jobs);
    const auto scan = [&](auto kernel, int waves) { kernel<<<grid, kScan * waves, 0, s>>>(a, share, ws, cols); };
    if (share.segments <= 4) scan(k_scan<1, 4>, 1);
    else if (share.segments <= 16) scan(k_scan<4, 4>, 4);
    else if (share.segments <= 64) scan(k_scan<4, 16>, 4);
    else scan(k_scan<16, 16>, 16);
  }
  launch<E>(how, a, share, ws, kMain, a.roles, K, V, s);
  return hipGetLastError();
}
template <typename E> hipError_t step(const LinearStep& a, hipStream_t s) {
  const unsigned n = (unsigned)(a.P * a.B * a.H);
  if (a.K * a.V <= 1024) k_step<E, 1><<<n, 64, 0, s>>>(a);
  else k_step<E, 4><<<n, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace linear
}  // namespace

int64_t linear_workspace_bytes(int64_t P, int64_t B, int64_t T, int64_t H, int64_t K, int64_t V, int dtype, bool backward) {
  using namespace linear;
  const Share share = share_of(P * B * H, T, (int)K, (int)V, dtype, backward);
  if (share.segments == 1) return 0;
  return ((int64_t)share.jobs * share.segments * P * B * H * (K * V + 1) * 4 + 255) / 256 * 256;
}

hipError_t launch_linear(const LinearArgs& a, int dtype, void* ws, hipStream_t s) {
  return dtype == POP_F32 ? linear::run<float>(a, dtype, (float*)ws, s) : dtype == POP_BF16 ? linear::run<__bf16>(a, dtype, (float*)ws, s) : linear::run<_Float16>(a, dtype, (float*)ws, s);
}
hipError_t launch_linear_step(const LinearStep& a, int dtype, hipStream_t s) {
  return dtype == POP_F32 ? linear::step<float>(a, s) : dtype == POP_BF16 ? linear::step<__bf16>(a, s) : linear::step<_Float16>(a, s);
}

}  // namespace pop
