// Linear attention with a decay for each head over sequences, its backward pass, and single steps (operators.h).
//
// HEADER
#include <hip/hip_runtime.h>
#include "operators.h"

namespace pop {
namespace {
namespace linear {

#ifndef POP_OCC
#define POP_OCC 2
#endif
#ifndef POP_C
#define POP_C 32
#endif
constexpr int kThreads = 256, kMost = POP_LINEAR_MAX_DIM;

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

// Operands of a product are sums of bf16 parts: an array's values exactly (kIn of them), a computed operand (a weight, a state, a
// value times its decay) to 24 bits for fp32 arrays and to 16 for 16-bit ones, whose own values have 8 or 11.
template <typename E> struct Parts { static constexpr int kIn = 2, kOf = 2; };
template <> struct Parts<__bf16> { static constexpr int kIn = 1, kOf = 2; };
template <> struct Parts<float> { static constexpr int kIn = 3, kOf = 3; };

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
// c + a b: all products of parts but those below the last part's rounding.
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

__device__ inline void sync_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// How a call's sequences are shared: `segments` of `per` chunks each, which go from the states that k_scan leaves.
struct Share { int chunks, per, segments, jobs; };
enum { kMain = 0, kStates = 1 };

// How a call's arrays are reached.  kWide: vectors of 16 bytes of q and k, four columns of o at a time, elements of v; kNarrow: elements, as
// rows lie at odd places; kAny: elements by addresses of 64 bits, for steps further apart than 32 bits reach, and steps that lie
// over each other.
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

// The channel that row 4 g + i of tile d of the state stands for: tiles 2 n and 2 n + 1 share 32 channels so that what a lane has of both is
// eight in a row, as the operands from LDS have them.
__device__ inline int channel_of(int d, int g, int i) { return 32 * (d / 2) + 8 * g + 4 * (d % 2) + i; }

// C steps of an array's channels: the threads of the workgroup take vectors of 16 bytes in turn.  Row r of a chunk is its step r, from the
// end in reverse.
template <typename E, int KB, int NW, int C, int HOW> struct Tile {
  static constexpr int kVec = 16 / sizeof(E), kAcross = 32 * KB / kVec, kAll = C * kAcross, kEach = (kAll + 64 * NW - 1) / (64 * NW);
  static constexpr int kStride = 32 * KB + 8, kPlane = C * kStride, kIn = Parts<E>::kIn;
  u32x4 v[kEach];
  static __device__ inline int row(int i) { return (int)(threadIdx.x + i * 64 * NW) / kAcross; }
  static __device__ inline int channel(int i) { return (int)(threadIdx.x + i * 64 * NW) % kAcross * kVec; }
  __device__ inline void load(const Steps<E, C, HOW>& a, int n, bool reverse) {
    const auto r = a.chunk(n);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int m = reverse ? C - 1 - row(i) : row(i);
      if constexpr (HOW == kWide) {
        v[i] = __builtin_amdgcn_raw_buffer_load_b128(r, a.offset(m, channel(i)), 0, 0);
      } else {
        E e[kVec];
#pragma unroll
        for (int k = 0; k < kVec; ++k) e[k] = a.element(r, n, m, channel(i) + k);
        __builtin_memcpy(&v[i], e, 16);
      }
    }
  }
  // Into LDS, part by part.  Returns whether all values are finite.
  __device__ inline bool store(unsigned short* plane) const {
    unsigned bad = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (kAll % (64 * NW) != 0 && row(i) >= C) break;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const unsigned w = v[i][d];
        if constexpr (sizeof(E) == 4) bad |= (w & 0x7f800000u) + 0x00800000u;
        else if constexpr (kIn == 1) bad |= (w & 0x7f807f80u) + 0x00800080u;
        else bad |= (w & 0x7c007c00u) + 0x04000400u;
      }
      unsigned short* to = plane + row(i) * kStride + channel(i);
      if constexpr (kIn == 1) {
        *(u32x4*)to = v[i];
      } else if constexpr (sizeof(E) == 4) {
        unsigned lo[3], hi[3];
        split<3>(__uint_as_float(v[i][0]), __uint_as_float(v[i][1]), lo);
        split<3>(__uint_as_float(v[i][2]), __uint_as_float(v[i][3]), hi);
#pragma unroll
        for (int n = 0; n < 3; ++n) *(u32x2*)(to + n * kPlane) = u32x2{lo[n], hi[n]};
      } else {
        u32x4 p[2];
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          typedef _Float16 pair __attribute__((ext_vector_type(2)));
          const unsigned w = v[i][d];                                // (of an element in its place the cast takes the first)
          const pair x = __builtin_bit_cast(pair, w);
          unsigned part[2];
          split<2>((float)x[0], (float)x[1], part);
          p[0][d] = part[0];
          p[1][d] = part[1];
        }
        *(u32x4*)to = p[0];
        *(u32x4*)(to + kPlane) = p[1];
      }
    }
    return (bad & (sizeof(E) == 4 ? 0x80000000u : 0x80008000u)) == 0;
  }
  // Rows 16 tile .. of 32 channels as an operand: a lane has channels 8 g .. 8 g + 7.
  static __device__ inline Operand<kIn> rows(const unsigned short* plane, int tile, int kb, int lane) {
    Operand<kIn> o;
    const unsigned short* from = plane + (16 * tile + (lane & 15)) * kStride + 32 * kb + 8 * (lane >> 4);
#pragma unroll
    for (int n = 0; n < kIn; ++n) o.part[n] = *(const u32x4*)(from + n * kPlane);
    return o;
  }
  // The channels of half `d % 2` of block d / 2 (channel_of) of 32 rows as an operand: four rows of four times four channels, turned over by
  // the read.
  static __device__ inline Operand<kIn> channels(unsigned short* plane, int block, int d, int lane) {
    Operand<kIn> o;
    unsigned short* from = plane + (32 * block + 4 * (lane >> 4) + (lane & 15) / 4) * kStride + channel_of(d, lane & 3, 0);
#pragma unroll
    for (int n = 0; n < kIn; ++n) {
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((POP_LDS s16x4*)(from + n * kPlane));
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((POP_LDS s16x4*)(from + n * kPlane + 16 * kStride));
      const u32x2 x = __builtin_bit_cast(u32x2, a), y = __builtin_bit_cast(u32x2, b);
      o.part[n] = u32x4{x[0], x[1], y[0], y[1]};
    }
    return o;
  }
};

__device__ inline float power(float log2_decay, int n) { return __builtin_amdgcn_exp2f((float)n * log2_decay); }
__device__ inline bool not_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }
__device__ inline bool any_lane(bool v) { return __builtin_amdgcn_ballot_w64(v) != 0; }

// A wavefront has 16 VT of the state's columns, the workgroup those of NW wavefronts.
template <typename E, int KB, int NW, int VT, int C, int HOW>
__global__ void __launch_bounds__(64 * NW, POP_OCC) k_chunks(LinearArgs a, Share share, float* ws, int mode) {
  typedef Tile<E, KB, NW, C, HOW> T;
  typedef Steps<E, C, HOW> Array;
  constexpr int kIn = Parts<E>::kIn, kOf = Parts<E>::kOf, kTiles = C / 16, kBlocks = C / 32;
  static_assert(C == 32, "starts of episodes are the bits of a word");
  __shared__ __attribute__((aligned(16))) unsigned short lds[2 * kIn * T::kPlane];
  __shared__ int bad_keys[2];
  unsigned short *const keys = lds, *const queries = lds + kIn * T::kPlane;
  const LinearRole& role = a.role[blockIdx.z];
  const int col = blockIdx.x, seg = blockIdx.y, h = col % a.H, row = col / a.H, b = row % a.B, p = row / a.B;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, at = lane & 15, K = role.K, V = role.V;
  const bool reverse = role.reverse, states = mode == kStates;
  const int len = a.lengths ? min(max(a.lengths[row], 0), a.T) : a.T;
  const uint8_t* reset = a.reset.data ? (const uint8_t*)a.reset.data + p * a.reset.agent + b * a.reset.row : nullptr;
  const float l2 = log_decay_of(a.log_decay, p * a.H + h) * 1.44269504f, lambda = power(l2, 1);
  const int before = reverse ? 0 : 1, behind = reverse ? 1 : 0;     // factors of the state on its way in and out, beside those between rows
  const int segment = reverse ? share.segments - 1 - seg : seg, from = min(segment * share.per, share.chunks), until = min(from + share.per, share.chunks);
  const int start = from * C, end = min(until * C, a.T), n_chunks = max(0, (min(end, len) - start + C - 1) / C);
  const int first_t = start + (reverse ? max(n_chunks - 1, 0) * C : 0);
  Array q(role.q, p, b, h, K, first_t, reverse), k(role.k, p, b, h, K, first_t, reverse), v(role.v, p, b, h, V, first_t, reverse), o(role.o, p, b, h, V, first_t, reverse);
  const int first_column = 16 * VT * wave;                           // this lane's columns: first_column + 16 c + at
  const bool idle = first_column >= V;                               // a wave with no columns loads with the others

  // the state: S[c][d][i] is channel channel_of(d, g, i) of column c
  f32x4 S[VT][2 * KB];
  bool tainted = false;
  {
    const float* first = states ? nullptr : share.segments > 1 ? ws : role.first;
    int64_t base = (int64_t)col * K * V;
    int along_k = role.first_k, along_v = role.first_v;
    if (share.segments > 1) {
      const int job = blockIdx.z == 2 ? 1 : blockIdx.z;              // role 2 takes the states of role 1, transposed
      base += ((int64_t)job * share.segments + seg) * gridDim.x * K * V;
      along_k = blockIdx.z == 2 ? 1 : V;
      along_v = blockIdx.z == 2 ? K : 1;
    }
#pragma unroll
    for (int c = 0; c < VT; ++c)
#pragma unroll
      for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row_k = channel_of(d, g, i), column = first_column + 16 * c + at;
          S[c][d][i] = first && row_k < K && column < V ? first[base + row_k * along_k + column * along_v] : 0.0f;
          tainted |= not_finite(S[c][d][i]);
        }
    tainted = any_lane(tainted);
  }

  // Weights of pairs, row `at` of a tile and row 4 g + j of another: the same tile, one in front; further ones by a power for the tile.
  // Weights of the state on its way in and out.
  const float both = role.read * role.write, whole = power(l2, C);
  float here[4], there[4], tiles[kTiles], into[kTiles], outof[kTiles][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    here[j] = both * power(l2, max(at - 4 * g - j, 0));
    there[j] = both * power(l2, 16 + at - 4 * g - j);
  }
#pragma unroll
  for (int n = 0; n < kTiles; ++n) {
    tiles[n] = power(l2, 16 * n);
    into[n] = role.read * power(l2, 16 * n + at + before);
#pragma unroll
    for (int j = 0; j < 4; ++j) outof[n][j] = role.write * power(l2, C - 1 - (16 * n + 4 * g + j) + behind);
  }

  T next_k, next_q;
  E next_v[VT][C / 4];
  uint8_t next_cut = 0;
  const auto load = [&](int n) {
    const int t = start + (reverse ? n_chunks - 1 - n : n) * C, count = min(C, len - t);
    next_k.load(k, count, reverse);
    if (!states) next_q.load(q, count, reverse);
    const auto r = v.chunk(count);
#pragma unroll
    for (int c = 0; c < VT; ++c)
#pragma unroll
      for (int j = 0; j < C / 4; ++j) {
        const int s = 16 * (j / 4) + 4 * g + j % 4, m = reverse ? C - 1 - s : s, column = first_column + 16 * c + at;
        next_v[c][j] = v.element(r, count, m, column);
      }
    k.now += k.hop;
    q.now += q.hop;
    v.now += v.hop;
    if (reset) {
      const int m = reverse ? C - lane : lane;                       // in reverse what leads from the step behind to row `lane`
      next_cut = lane < C && t + m < len && m < count + (reverse ? 1 : 0) ? reset[(int64_t)(t + m) * a.reset.step] : 0;
    }
  };
  if (n_chunks > 0) load(0);
  if (threadIdx.x == 0) bad_keys[0] = 0;
  bool any_cut = false;

  for (int n = 0; n < n_chunks; ++n) {
    const int t = start + (reverse ? n_chunks - 1 - n : n) * C, count = min(C, len - t);
    if (n > 0) o.now += o.hop;
    sync_lds();                                                      // the chunk before has been read
    if (!next_k.store(keys)) bad_keys[n & 1] = 1;
    if (!states) next_q.store(queries);
    const unsigned cuts = (unsigned)__builtin_amdgcn_ballot_w64(next_cut != 0);
    f32x4 value[VT][kTiles];
    float zero = 0.0f;                                               // but where a value is not finite
#pragma unroll
    for (int c = 0; c < VT; ++c)
#pragma unroll
      for (int j = 0; j < C / 4; ++j) {
        value[c][j / 4][j % 4] = (float)next_v[c][j];
        zero = fmaf((float)next_v[c][j], 0.0f, zero);
      }
    sync_lds();
    if (n + 1 < n_chunks) load(n + 1);
    const bool slow = __builtin_amdgcn_readfirstlane(bad_keys[n & 1]) != 0 || any_lane(zero != 0.0f) || tainted;
    if (threadIdx.x == 0) bad_keys[(n + 1) & 1] = 0;
    any_cut |= cuts != 0;
    if (idle) continue;

    if (__builtin_expect(slow, 0)) {
      // something here is not finite, and a product with a weight of zero would carry it where it does not belong: step by step
      tainted = false;
      const E *qs = linear::at<E>(role.q, p, b, h), *ks = linear::at<E>(role.k, p, b, h), *vs = linear::at<E>(role.v, p, b, h);
      E* os = (E*)linear::at<E>(role.o, p, b, h);
#pragma unroll 1
      for (int r = reverse ? C - count : 0; r < (reverse ? C : count); ++r) {
        const int64_t s = t + (reverse ? C - 1 - r : r);
        const bool cut = cuts >> r & 1;
        const int g = here_only(lane >> 4), at = here_only(lane & 15);
#pragma unroll
        for (int c = 0; c < VT; ++c) {
          const int column = first_column + 16 * c + at;
          const float vr = column < V ? (float)vs[s * role.v.step + column] * role.write : 0.0f;
          float sum = 0.0f;
#pragma unroll
          for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int kr = channel_of(d, g, i);
              if (kr < K) {
                const float x = fmaf((float)ks[s * role.k.step + kr], vr, cut ? 0.0f : reverse ? S[c][d][i] : lambda * S[c][d][i]);
                if (!states) sum = fmaf((float)qs[s * role.q.step + kr], x, sum);
                S[c][d][i] = reverse ? lambda * x : x;
              }
            }
          sum += __shfl_xor(sum, 16);
          sum += __shfl_xor(sum, 32);
          if (!states && g == 0 && column < V) os[s * role.o.step + column] = (E)(sum * role.read);
        }
      }
#pragma unroll
      for (int c = 0; c < VT; ++c)
#pragma unroll
        for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) tainted |= not_finite(S[c][d][i]);
      tainted = any_lane(tainted);
      continue;
    }

    const bool regular = cuts == 0 && count == C;
    const auto starts = [&](int r) { return __popc(cuts & ((2u << here_only(r)) - 1)); };   // episodes that start at rows 0 .. r
    const int all_starts = __popc(cuts);

    if (!states) {
      Operand<kIn> values[VT][kBlocks];
      Operand<kOf> memory[VT][KB];
#pragma unroll
      for (int c = 0; c < VT; ++c) {
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) values[c][s] = operand<kIn>(value[c][2 * s], value[c][2 * s + 1]);
#pragma unroll
        for (int d = 0; d < KB; ++d) memory[c][d] = operand<kOf>(S[c][2 * d], S[c][2 * d + 1]);
      }
      const auto r = o.chunk(count);
#pragma unroll
      for (int tile = 0; tile < kTiles; ++tile) {
        Operand<kIn> query[KB];
        f32x4 out[VT];                                               // rows: columns 4 g + i of 16; column: row `at` of the tile
#pragma unroll
        for (int c = 0; c < VT; ++c) out[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int d = 0; d < KB; ++d) {
          query[d] = T::rows(queries, tile, d, lane);
#pragma unroll
          for (int c = 0; c < VT; ++c) out[c] = product(memory[c][d], query[d], out[c]);
        }
        const int i = 16 * tile + at;
        int mine = 0;
        float f = into[tile];
        if (!regular) {
          mine = starts(i);
          if (reverse) f = role.read * power(l2, max(here_only(i) - (C - count), 0));
        }
#pragma unroll
        for (int c = 0; c < VT; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) out[c][e] = mine == 0 ? out[c][e] * f : 0.0f;
#pragma unroll
        for (int block = 0; block <= tile / 2; ++block) {
          f32x4 weight[2];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int other = 2 * block + half;
            f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
            if (other <= tile) {
#pragma unroll
              for (int d = 0; d < KB; ++d) w = product(T::rows(keys, other, d, lane), query[d], w);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (other == tile) w[j] = 4 * g + j <= at ? w[j] * here[j] : 0.0f;
                else w[j] *= other + 1 == tile ? there[j] : there[j] * tiles[tile - other - 1];
              }
              if (!regular)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = starts(16 * other + 4 * g + j) == mine ? w[j] : 0.0f;
            }
            weight[half] = w;
          }
          const Operand<kOf> weights = operand<kOf>(weight[0], weight[1]);
#pragma unroll
          for (int c = 0; c < VT; ++c) out[c] = product(values[c][block], weights, out[c]);
        }
        const int m = reverse ? C - 1 - i : i;
#pragma unroll
        for (int c = 0; c < VT; ++c) {
          typedef E Four __attribute__((ext_vector_type(4)));
          const Four x = {(E)out[c][0], (E)out[c][1], (E)out[c][2], (E)out[c][3]};
          const int column = first_column + 16 * c + 4 * g;
          if constexpr (HOW == kWide) {
            if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), r, o.offset(m, column), 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, x), r, o.offset(m, column), 0, 0);
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

    float keep = whole;
    if (!regular) keep = power(l2, count);
#pragma unroll
    for (int c = 0; c < VT; ++c) {
      Operand<kOf> faded[kBlocks];
#pragma unroll
      for (int s = 0; s < kBlocks; ++s) {
        f32x4 x[2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = 32 * s + 16 * (j / 4) + 4 * g + j % 4;
          float f = outof[2 * s + j / 4][j % 4];
          if (!regular) {
            if (!reverse) f = role.write * power(l2, max(count - 1 - here_only(r), 0));
            f = starts(r) == all_starts ? f : 0.0f;
          }
          x[j / 4][j % 4] = value[c][2 * s + j / 4][j % 4] * f;
        }
        faded[s] = operand<kOf>(x[0], x[1]);
      }
#pragma unroll
      for (int d = 0; d < 2 * KB; ++d) {
        f32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = all_starts == 0 ? S[c][d][i] * keep : 0.0f;
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) x = product(T::channels(keys, s, d, lane), faded[s], x);
        S[c][d] = x;
      }
    }
  }

#pragma unroll
  for (int c = 0; c < VT; ++c) {
    const int column = first_column + 16 * c + at;
    if (!states && column < V)
      for (int t = max(start, len) + g; t < end; t += 4) ((E*)linear::at<E>(role.o, p, b, h))[t * role.o.step + column] = (E)0.0f;
  }
  const bool last = seg == share.segments - 1;
  float* to = states ? ws + (((int64_t)blockIdx.z * share.segments + seg) * gridDim.x + col) * K * V : last && role.last ? role.last + (int64_t)col * K * V : nullptr;
  if (!to) return;
  const bool cut = !states && reverse && len > 0 && reset && reset[0];
#pragma unroll
  for (int c = 0; c < VT; ++c)
#pragma unroll
    for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row_k = channel_of(d, g, i), column = first_column + 16 * c + at;
        if (row_k < K && column < V) to[row_k * V + column] = cut ? 0.0f : S[c][d][i];
      }
  if (states && threadIdx.x == 0) {
    float* factor = ws + (int64_t)share.jobs * share.segments * gridDim.x * K * V;
    factor[((int64_t)blockIdx.z * share.segments + seg) * gridDim.x + col] = any_cut ? -1.0f : power(l2, max(0, min(end, len) - start));
  }
}

// The states in front of the segments, in the places of what the segments add to them.  A negative factor: nothing of the state in front
// is left.
__global__ void __launch_bounds__(kThreads) k_scan(LinearArgs a, Share share, float* ws, int cols) {
  const LinearRole& role = a.role[blockIdx.y];
  const int64_t size = (int64_t)role.K * role.V, n = cols * size, i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const int col = (int)(i / size), e = (int)(i % size);
  float* at = ws + (int64_t)blockIdx.y * share.segments * n + i;
  const float* factor = ws + (int64_t)share.jobs * share.segments * n + (int64_t)blockIdx.y * share.segments * cols + col;
  float s = role.first ? role.first[col * size + e / role.V * role.first_k + e % role.V * role.first_v] : 0.0f;
  float add = at[0], f = factor[0];
  for (int k = 0; k < share.segments; ++k) {
    const float add_now = add, f_now = f;
    if (k + 1 < share.segments) {
      add = at[(k + 1) * n];
      f = factor[(int64_t)(k + 1) * cols];
    }
    at[k * n] = s;
    s = f_now < 0.0f ? add_now : fmaf(f_now, s, add_now);
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

// Sequences are cut into segments where there are too few of them: the segments' own states first, then those in front of them.
constexpr int kChunk = POP_C, kWorkgroups = 1024, kLeast = 4, kMostSegments = 4096;
template <typename E> constexpr int chunk_of(int K) { return kChunk; }
Share share_of(int64_t cols, int64_t T, int chunk, bool backward) {
  const int64_t chunks = (T + chunk - 1) / chunk, roles = backward ? 3 : 1;
  int64_t want = kWorkgroups / (cols * roles);
  if (want > kMostSegments) want = kMostSegments;
  if (want > chunks / kLeast) want = chunks / kLeast;
  if (want <= 1) return {(int)chunks, (int)chunks, 1, 0};
  const int64_t per = (chunks + want - 1) / want;
  return {(int)chunks, (int)per, (int)((chunks + per - 1) / per), backward ? 2 : 1};
}

#ifndef POP_VT
#define POP_VT 1
#endif
template <typename E, int KB, int NW, int HOW> void chunks(const LinearArgs& a, const Share& share, float* ws, int mode, dim3 grid, hipStream_t s) {
  constexpr int VT = NW >= 2 * POP_VT ? POP_VT : 1;
  k_chunks<E, KB, NW / VT, VT, kChunk, HOW><<<grid, 64 * NW / VT, 0, s>>>(a, share, ws, mode);
}
template <typename E, int KB, int HOW> void launch(const LinearArgs& a, const Share& share, float* ws, int mode, dim3 grid, int V, hipStream_t s) {
  if (V > 64) chunks<E, KB, 8, HOW>(a, share, ws, mode, grid, s);
  else if (V > 32) chunks<E, KB, 4, HOW>(a, share, ws, mode, grid, s);
  else chunks<E, KB, 2, HOW>(a, share, ws, mode, grid, s);
}
template <typename E, int HOW> void launch(const LinearArgs& a, const Share& share, float* ws, int mode, dim3 grid, int K, int V, hipStream_t s) {
  if (K <= 32) launch<E, 1, HOW>(a, share, ws, mode, grid, V, s);
  else if (K <= 64) launch<E, 2, HOW>(a, share, ws, mode, grid, V, s);
  else launch<E, 4, HOW>(a, share, ws, mode, grid, V, s);
}
template <typename E> void launch(int how, const LinearArgs& a, const Share& share, float* ws, int mode, dim3 grid, int K, int V, hipStream_t s) {
  if (how == kWide) launch<E, kWide>(a, share, ws, mode, grid, K, V, s);
  else if (how == kNarrow) launch<E, kNarrow>(a, share, ws, mode, grid, K, V, s);
  else chunks<E, POP_LINEAR_MAX_DIM / 32, POP_LINEAR_MAX_DIM / 16, kAny>(a, share, ws, mode, grid, s);
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
    if (!aligned(r.q, r.K, 16 / sizeof(E)) || !aligned(r.k, r.K, 16 / sizeof(E)) || !aligned(r.o, r.V, 4)) how = kNarrow;
  }
  return how;
}
template <typename E> hipError_t run(const LinearArgs& a, float* ws, hipStream_t s) {
  const int64_t cols = (int64_t)a.P * a.B * a.H;
  // roles of one shape go together
  const int K = a.role[0].K > a.role[0].V ? a.role[0].K : a.role[0].V;
  const Share share = share_of(cols, a.T, chunk_of<E>(a.roles > 1 ? K : a.role[0].K), a.roles > 1);
  const int kk = a.roles > 1 ? K : a.role[0].K, vv = a.roles > 1 ? K : a.role[0].V;
  const int how = how_of<E>(a);
  if (share.segments > 1) {
    launch<E>(how, a, share, ws, kStates, dim3((unsigned)cols, share.segments, share.jobs), kk, vv, s);
    k_scan<<<dim3((unsigned)((cols * a.role[0].K * a.role[0].V + kThreads - 1) / kThreads), share.jobs), kThreads, 0, s>>>(a, share, ws, (int)cols);
  }
  launch<E>(how, a, share, ws, kMain, dim3((unsigned)cols, share.segments, a.roles), kk, vv, s);
  return hipGetLastError();
}
template <typename E> hipError_t step(const LinearStep& a, hipStream_t s) {
  k_step<E><<<(unsigned)(a.P * a.B * a.H), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace linear
}  // namespace

int64_t linear_workspace_bytes(int64_t P, int64_t B, int64_t T, int64_t H, int64_t K, int64_t V, int64_t element, bool backward) {
  using namespace linear;
  const int64_t wide = backward && V > K ? V : K;
  const Share share = share_of(P * B * H, T, element == 4 ? chunk_of<float>((int)wide) : kChunk, backward);
  if (share.segments == 1) return 0;
  return ((int64_t)share.jobs * share.segments * P * B * H * (K * V + 1) * 4 + 255) / 256 * 256;
}

hipError_t launch_linear(const LinearArgs& a, int dtype, void* ws, hipStream_t s) {
  return dtype == POP_F32 ? linear::run<float>(a, (float*)ws, s) : dtype == POP_BF16 ? linear::run<__bf16>(a, (float*)ws, s) : linear::run<_Float16>(a, (float*)ws, s);
}
hipError_t launch_linear_step(const LinearStep& a, int dtype, hipStream_t s) {
  return dtype == POP_F32 ? linear::step<float>(a, s) : dtype == POP_BF16 ? linear::step<__bf16>(a, s) : linear::step<_Float16>(a, s);
}

}  // namespace pop
