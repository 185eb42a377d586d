// Linear attention with a decay for each head over sequences, its backward pass, and single steps (operators.h).
//
// HEADER
#include <hip/hip_runtime.h>
#include "operators.h"

namespace pop {
namespace {
namespace linear {

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
// of the 32 that are summed over.  Their order is free as long as both operands have the same, and in this one two results lie one
// under the other (rows 4 g + j of each) are an operand as they are.
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

// Rows of a chunk: row r is step `first` + r * `dir` of the sequence.
struct Rows { int first, dir, n; };

// C rows of an array's K channels: lane `t` of the workgroup takes the vectors t, t + 64 NW, ...
template <typename E, int KB, int NW, int C> struct Tile {
  static constexpr int kVec = 16 / sizeof(E), kAcross = 32 * KB / kVec, kAll = C * kAcross, kEach = (kAll + 64 * NW - 1) / (64 * NW), kStride = 32 * KB + 8, kPlane = C * kStride;
  static constexpr int kIn = Parts<E>::kIn;
  u32x4 v[kEach];
  __device__ inline void load(const E* base, int64_t step, const Rows& rows, int K, bool wide) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = threadIdx.x + i * 64 * NW, r = at / kAcross, c = at % kAcross * kVec;
      const E* from = base + (int64_t)(rows.first + min(r, rows.n - 1) * rows.dir) * step;
      if (wide) {
        v[i] = *(const u32x4*)(from + (c < K ? c : 0));
      } else {
        E e[kVec];
#pragma unroll
        for (int k = 0; k < kVec; ++k) e[k] = from[min(c + k, K - 1)];
        __builtin_memcpy(&v[i], e, 16);
      }
    }
  }
  // Zeros in the place of what does not exist; then into LDS.  Returns whether all values are finite.
  __device__ inline bool store(unsigned short* plane, const Rows& rows, int K) {
    unsigned bad = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = threadIdx.x + i * 64 * NW, r = at / kAcross, c = at % kAcross * kVec;
      const int exist = r < rows.n ? K - c : 0;
      if (kAll % (64 * NW) != 0 && at >= kAll) break;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        constexpr int kWord = 4 / sizeof(E);
        unsigned w = v[i][d];
        if (kWord == 1) w = d < exist ? w : 0u;
        else w = 2 * d + 1 < exist ? w : 2 * d < exist ? w & 0xffffu : 0u;
        v[i][d] = w;
        if constexpr (sizeof(E) == 4) bad |= (w & 0x7f800000u) == 0x7f800000u;
        else if constexpr (kIn == 1) bad |= ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
        else bad |= ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
      }
      unsigned short* to = plane + r * kStride + c;
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
    return bad == 0;
  }
  // Rows 16 tile .. of 32 channels as an operand.
  static __device__ inline Operand<kIn> rows(const unsigned short* plane, int tile, int kb, int lane) {
    Operand<kIn> o;
    const unsigned short* from = plane + (16 * tile + (lane & 15)) * kStride + 32 * kb + 4 * (lane >> 4);
#pragma unroll
    for (int n = 0; n < kIn; ++n) {
      const u32x2 a = *(const u32x2*)(from + n * kPlane), b = *(const u32x2*)(from + n * kPlane + 16);
      o.part[n] = u32x4{a[0], a[1], b[0], b[1]};
    }
    return o;
  }
  // Channels 16 tile .. of 32 rows as an operand: four rows of 16 channels, turned over by the read.
  static __device__ inline Operand<kIn> channels(unsigned short* plane, int block, int tile, int lane) {
    Operand<kIn> o;
    unsigned short* from = plane + (32 * block + 4 * (lane >> 4) + (lane & 15) / 4) * kStride + 16 * tile + (lane & 3) * 4;
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

template <typename E, int KB, int NW, int C>
__global__ void __launch_bounds__(64 * NW) k_chunks(LinearArgs a, Share share, float* ws, int mode) {
  typedef Tile<E, KB, NW, C> T;
  constexpr int kIn = Parts<E>::kIn, kOf = Parts<E>::kOf, kTiles = C / 16, kBlocks = C / 32;
  __shared__ __attribute__((aligned(16))) unsigned short lds[2 * kIn * T::kPlane];
  __shared__ int bad_keys[2];
  unsigned short *const keys = lds, *const queries = lds + kIn * T::kPlane;
  const LinearRole& role = a.role[blockIdx.z];
  const int col = blockIdx.x, seg = blockIdx.y, h = col % a.H, row = col / a.H, b = row % a.B, p = row / a.B;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, at = lane & 15, K = role.K, V = role.V;
  const bool reverse = role.reverse, states = mode == kStates;
  const int len = a.lengths ? min(max(a.lengths[row], 0), a.T) : a.T;
  const uint8_t* reset = a.reset.data ? (const uint8_t*)a.reset.data + p * a.reset.agent + b * a.reset.row : nullptr;
  const E* const q = linear::at<E>(role.q, p, b, h);
  const E* const k = linear::at<E>(role.k, p, b, h);
  const E* const v = linear::at<E>(role.v, p, b, h);
  E* const o = (E*)linear::at<E>(role.o, p, b, h);
  const float l2 = log_decay_of(a.log_decay, p * a.H + h) * 1.44269504f, lambda = power(l2, 1);
  const int before = reverse ? 0 : 1, behind = reverse ? 1 : 0;     // factors of the state on its way in and out, beside those between rows
  const int segment = reverse ? share.segments - 1 - seg : seg, from = min(segment * share.per, share.chunks), until = min(from + share.per, share.chunks);
  const int start = from * C, end = min(until * C, a.T), n_chunks = max(0, (min(end, len) - start + C - 1) / C);
  const int column = 16 * wave + at, own = min(column, V - 1);       // of this lane
  const bool idle = 16 * wave >= V;                                  // a wave with no columns loads with the others
  constexpr auto aligned = [](const pop_heads& s, int n) {
    return (uintptr_t)s.data % (n * sizeof(E)) == 0 && s.agent % n == 0 && s.row % n == 0 && s.step % n == 0 && s.head % n == 0;
  };
  const bool wide_k = K % T::kVec == 0 && aligned(role.k, T::kVec), wide_q = K % T::kVec == 0 && aligned(role.q, T::kVec);
  const bool wide_o = aligned(role.o, 4);

  // the state: S[d] has rows 16 d + 4 g + i, column `column`
  f32x4 S[2 * KB];
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
    for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row_k = 16 * d + 4 * g + i;
        S[d][i] = first && row_k < K && column < V ? first[base + row_k * along_k + column * along_v] : 0.0f;
        tainted |= not_finite(S[d][i]);
      }
    tainted = __builtin_amdgcn_ballot_w64(tainted) != 0;
  }

  // weights of pairs: row i of a tile, row s = 4 g + j of a tile `n` before it
  float pair[kTiles][4], into[kTiles], outof[kBlocks][8];
  const float both = role.read * role.write;
#pragma unroll
  for (int n = 0; n < kTiles; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) pair[n][j] = both * power(l2, max(16 * n + at - 4 * g - j, 0));
#pragma unroll
  for (int n = 0; n < kTiles; ++n) into[n] = role.read * power(l2, 16 * n + at + before);
#pragma unroll
  for (int n = 0; n < kBlocks; ++n)
#pragma unroll
    for (int j = 0; j < 8; ++j) outof[n][j] = role.write * power(l2, C - 1 - (32 * n + 16 * (j / 4) + 4 * g + j % 4) + behind);
  const float whole = power(l2, C);

  T next_k, next_q;
  E next_v[C / 4];
  uint8_t next_cut = 0;
  Rows rows = {0, 0, 1};
  const auto rows_of = [&](int n) {
    const int t = start + (reverse ? n_chunks - 1 - n : n) * C, count = min(C, len - t);
    return Rows{reverse ? t + count - 1 : t, reverse ? -1 : 1, count};
  };
  const auto load = [&](const Rows& r) {
    next_k.load(k, role.k.step, r, K, wide_k);
    if (!states) next_q.load(q, role.q.step, r, K, wide_q);
#pragma unroll
    for (int j = 0; j < C / 4; ++j) {
      const int s = 16 * (j / 4) + 4 * g + j % 4;
      next_v[j] = v[(int64_t)(r.first + min(s, r.n - 1) * r.dir) * role.v.step + own];
    }
    if (reset) {
      const int t = r.first + min(lane, r.n - 1) * r.dir + (reverse ? 1 : 0);
      next_cut = lane < r.n && t < len ? reset[(int64_t)t * a.reset.step] : 0;
    }
  };
  if (n_chunks > 0) {
    rows = rows_of(0);
    load(rows);
  }
  if (threadIdx.x == 0) bad_keys[0] = 0;
  bool any_cut = false;

  for (int n = 0; n < n_chunks; ++n) {
    sync_lds();                                                      // the chunk before has been read
    if (!next_k.store(keys, rows, K)) bad_keys[n & 1] = 1;
    if (!states) next_q.store(queries, rows, K);
    const uint64_t cuts = __builtin_amdgcn_ballot_w64(next_cut != 0);
    f32x4 value[C / 16];
    bool bad = false;
#pragma unroll
    for (int j = 0; j < C / 4; ++j) {
      const float x = 16 * (j / 4) + 4 * g + j % 4 < rows.n ? (float)next_v[j] : 0.0f;
      value[j / 4][j % 4] = x;
      bad |= not_finite(x);
    }
    const Rows now = rows;
    sync_lds();
    if (n + 1 < n_chunks) {
      rows = rows_of(n + 1);
      load(rows);
    }
    const bool slow = bad_keys[n & 1] != 0 || __builtin_amdgcn_ballot_w64(bad) != 0 || tainted;
    if (threadIdx.x == 0) bad_keys[(n + 1) & 1] = 0;
    any_cut |= cuts != 0;
    if (idle) continue;

    if (__builtin_expect(slow, 0)) {
      // something here is not finite, and a product with a weight of zero would carry it where it does not belong: step by step
      for (int r = 0; r < now.n; ++r) {
        const int64_t t = now.first + r * now.dir;
        const bool cut = cuts >> r & 1;
        const float vr = (float)v[t * role.v.step + own] * role.write;
        float sum = 0.0f;
#pragma unroll
        for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int kr = 16 * d + 4 * g + i;
            if (kr < K) {
              const float s = fmaf((float)k[t * role.k.step + kr], vr, cut ? 0.0f : reverse ? S[d][i] : lambda * S[d][i]);
              if (!states) sum = fmaf((float)q[t * role.q.step + kr], s, sum);
              S[d][i] = reverse ? lambda * s : s;
            }
          }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (!states && g == 0 && column < V) o[t * role.o.step + column] = (E)(sum * role.read);
      }
      tainted = false;
#pragma unroll
      for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) tainted |= not_finite(S[d][i]);
      tainted = __builtin_amdgcn_ballot_w64(tainted) != 0;
      continue;
    }

    const bool regular = cuts == 0 && now.n == C;
    const auto starts = [&](int r) { return __popcll(cuts & ((2ull << r) - 1)); };          // episodes that start at rows 0 .. r
    const int all_starts = __popcll(cuts);

    if (!states) {
      Operand<kIn> values[kBlocks];
      Operand<kOf> memory[KB];
#pragma unroll
      for (int s = 0; s < kBlocks; ++s) values[s] = operand<kIn>(value[2 * s], value[2 * s + 1]);
#pragma unroll
      for (int d = 0; d < KB; ++d) memory[d] = operand<kOf>(S[2 * d], S[2 * d + 1]);
#pragma unroll
      for (int tile = 0; tile < kTiles; ++tile) {
        Operand<kIn> query[KB];
        f32x4 out = {0.0f, 0.0f, 0.0f, 0.0f};                        // rows: columns 4 g + i of the wave; column: row `at` of the tile
#pragma unroll
        for (int d = 0; d < KB; ++d) {
          query[d] = T::rows(queries, tile, d, lane);
          out = product(memory[d], query[d], out);
        }
        const int i = 16 * tile + at, mine = starts(i);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = regular || mine == 0 ? out[e] * into[tile] : 0.0f;
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
                w[j] *= pair[tile - other][j];
                if (other == tile) w[j] = 4 * g + j <= at ? w[j] : 0.0f;
              }
              if (!regular)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = starts(16 * other + 4 * g + j) == mine ? w[j] : 0.0f;
            }
            weight[half] = w;
          }
          out = product(values[block], operand<kOf>(weight[0], weight[1]), out);
        }
        if (i < now.n) {
          E* to = o + (int64_t)(now.first + i * now.dir) * role.o.step + 16 * wave + 4 * g;
          typedef E Four __attribute__((ext_vector_type(4)));
          if (wide_o && 16 * wave + 4 * g + 3 < V) {
            *(Four*)to = Four{(E)out[0], (E)out[1], (E)out[2], (E)out[3]};
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (16 * wave + 4 * g + e < V) to[e] = (E)out[e];
          }
        }
      }
    }

    Operand<kOf> faded[kBlocks];
    float keep = whole;
    if (!regular) keep = power(l2, now.n);
#pragma unroll
    for (int s = 0; s < kBlocks; ++s) {
      f32x4 x[2];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int r = 32 * s + 16 * (j / 4) + 4 * g + j % 4;
        float f = outof[s][j];
        if (!regular) f = r < now.n && starts(r) == all_starts ? role.write * power(l2, now.n - 1 - r + behind) : 0.0f;
        x[j / 4][j % 4] = value[2 * s + j / 4][j % 4] * f;
      }
      faded[s] = operand<kOf>(x[0], x[1]);
    }
#pragma unroll
    for (int d = 0; d < 2 * KB; ++d) {
      f32x4 c;
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = all_starts == 0 ? S[d][i] * keep : 0.0f;
#pragma unroll
      for (int s = 0; s < kBlocks; ++s) c = product(T::channels(keys, s, d, lane), faded[s], c);
      S[d] = c;
    }
  }

  if (!states && column < V && !idle)
    for (int t = max(start, len) + g; t < end; t += 4) o[(int64_t)t * role.o.step + column] = (E)0.0f;

  const bool last = seg == share.segments - 1;
  float* to = states ? ws + (((int64_t)blockIdx.z * share.segments + seg) * gridDim.x + col) * K * V : last && role.last ? role.last + (int64_t)col * K * V : nullptr;
  if (!to) return;
  const bool cut = !states && reverse && len > 0 && reset && reset[0];
#pragma unroll
  for (int d = 0; d < 2 * KB; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row_k = 16 * d + 4 * g + i;
      if (row_k < K && column < V) to[row_k * V + column] = cut ? 0.0f : S[d][i];
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
constexpr int kChunk = 64, kWorkgroups = 1024, kLeast = 4, kMostSegments = 4096;
template <typename E> constexpr int chunk_of(int K) { return sizeof(E) == 4 && K > 64 ? 32 : kChunk; }
Share share_of(int64_t cols, int64_t T, int chunk, bool backward) {
  const int64_t chunks = (T + chunk - 1) / chunk, roles = backward ? 3 : 1;
  int64_t want = kWorkgroups / (cols * roles);
  if (want > kMostSegments) want = kMostSegments;
  if (want > chunks / kLeast) want = chunks / kLeast;
  if (want <= 1) return {(int)chunks, (int)chunks, 1, 0};
  const int64_t per = (chunks + want - 1) / want;
  return {(int)chunks, (int)per, (int)((chunks + per - 1) / per), backward ? 2 : 1};
}

template <typename E, int KB, int NW> void chunks(const LinearArgs& a, const Share& share, float* ws, int mode, dim3 grid, hipStream_t s) {
  constexpr int C = chunk_of<E>(32 * KB);
  k_chunks<E, KB, NW, C><<<grid, 64 * NW, 0, s>>>(a, share, ws, mode);
}
template <typename E> void launch(const LinearArgs& a, const Share& share, float* ws, int mode, dim3 grid, int K, int V, hipStream_t s) {
  if (V > 64) {
    if (K <= 32) chunks<E, 1, 8>(a, share, ws, mode, grid, s);
    else if (K <= 64) chunks<E, 2, 8>(a, share, ws, mode, grid, s);
    else chunks<E, 4, 8>(a, share, ws, mode, grid, s);
  } else {
    if (K <= 32) chunks<E, 1, 4>(a, share, ws, mode, grid, s);
    else if (K <= 64) chunks<E, 2, 4>(a, share, ws, mode, grid, s);
    else chunks<E, 4, 4>(a, share, ws, mode, grid, s);
  }
}
template <typename E> hipError_t run(const LinearArgs& a, float* ws, hipStream_t s) {
  const int64_t cols = (int64_t)a.P * a.B * a.H;
  // roles of one shape go together
  const int K = a.role[0].K > a.role[0].V ? a.role[0].K : a.role[0].V;
  const Share share = share_of(cols, a.T, chunk_of<E>(a.roles > 1 ? K : a.role[0].K), a.roles > 1);
  const int kk = a.roles > 1 ? K : a.role[0].K, vv = a.roles > 1 ? K : a.role[0].V;
  if (share.segments > 1) {
    launch<E>(a, share, ws, kStates, dim3((unsigned)cols, share.segments, share.jobs), kk, vv, s);
    k_scan<<<dim3((unsigned)((cols * a.role[0].K * a.role[0].V + kThreads - 1) / kThreads), share.jobs), kThreads, 0, s>>>(a, share, ws, (int)cols);
  }
  launch<E>(a, share, ws, kMain, dim3((unsigned)cols, share.segments, a.roles), kk, vv, s);
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
