// Operators for populations of recurrent agents: what the boundary (op_api.hip) hands to the launch wrappers of
// k_recurrence.hip, k_linear.hip, k_clip.hip and k_orthogonalize.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "../../include/pop.h"

namespace pop {

// The message pop_last_error(NULL) returns on this thread (pop_api.hip); returns `code`.
int fail_thread(int code, const char* fmt, ...);

// ---- gated linear recurrence

constexpr int kRecurChunk = 128;     // steps between the states that forward leaves for backward

struct RecurArgs {
  int P, B, T, C;
  pop_sequence x, g, y, reset;       // single steps use no step strides
  const float *bias, *h0;
  const int32_t* lengths;
  float *h_last, *states;            // states: [P * B, chunks, C], the state before each chunk
  float* ws;
  // backward
  pop_sequence dy, dx, dg;
  const float* dh_last;
  float *dh0, *dbias;
  // single steps
  float* state;
  int n_slots;
  const int32_t* slots;
};

inline int64_t recur_chunks(int64_t T) { return (T + kRecurChunk - 1) / kRecurChunk; }
int64_t recur_workspace_floats(int64_t P, int64_t B, int64_t T, int64_t C, int64_t element);
hipError_t launch_recur_forward(const RecurArgs& a, int dtype, hipStream_t s);
hipError_t launch_recur_backward(const RecurArgs& a, int dtype, hipStream_t s);
hipError_t launch_recur_step(const RecurArgs& a, int dtype, hipStream_t s);

// ---- linear attention with a decay for each head

// o_t = `read` S_t^T q_t, S_t = lambda keep_t S_{t-1} + `write` k_t v_t^T from `first`.  In reverse time runs from the end and the
// factor of S lies behind step t instead of in front of it: S_t = lambda keep_{t+1} S_{t+1} + write k_t v_t^T.
struct LinearRole {
  pop_heads q, k, v, o;
  int K, V;                          // widths of q and k, of v and o
  int reverse;
  float read, write;
  const float* first;                // or NULL: zeros.  Element [i, j] of a state at i * first_k + j * first_v
  int first_k, first_v;
  float* last;                       // [i, j] at i * V + j; in reverse the gradient in front of step 0; or NULL
};
struct LinearArgs {
  int P, B, T, H;
  unsigned border;                   // (of the launch wrapper) what keys and queries stay below so that their products are in fp32's range
  const float* log_decay;            // [P, H] or NULL: zeros
  pop_sequence reset;
  const int32_t* lengths;
  int roles;
  LinearRole role[3];
};
struct LinearStep {
  int P, B, H, K, V;
  pop_heads q, k, v, o;              // no step strides
  pop_sequence reset;
  float scale;
  const float* log_decay;
  float* state;
  int n_slots;
  const int32_t* slots;
};
int64_t linear_workspace_bytes(int64_t P, int64_t B, int64_t T, int64_t H, int64_t K, int64_t V, int dtype, bool backward);
hipError_t launch_linear(const LinearArgs& a, int dtype, void* ws, hipStream_t s);
hipError_t launch_linear_step(const LinearStep& a, int dtype, hipStream_t s);

// ---- norms of gradients, clipping

constexpr int kClipPiece = 1 << 13;  // elements of one agent's part of a tensor that a workgroup takes at a time
inline int64_t clip_pieces(int64_t elements) { return (elements + kClipPiece - 1) / kClipPiece; }

struct ClipCall {
  int P, n;
  const pop_gradient* grads;
  double eps;
  const float* max_norm;             // NULL: norms only
  float* norms;                      // or NULL
};
int64_t clip_workspace_bytes(int64_t P, int n, const pop_gradient* grads);
hipError_t launch_clip(const ClipCall& c, void* ws, hipStream_t s);


// ---- orthogonalised updates

constexpr int kNsMaxSide = 16384;
constexpr float kSegmentGain = 0x1p11f;    // most that all steps together may multiply small singular values by for segments of three

struct NsLayer {                     // matrices of one shape
  int rows, cols, count;
  const void* g;                     // gradients, or the matrices to orthogonalise
  int64_t g_matrix, g_row;
  void* out;                         // orthogonalised matrices, of g's type; or NULL and
  int64_t out_matrix, out_row;
  float *momentum, *weight;          // momenta and weights to update
  int64_t m_matrix, m_row, w_matrix, w_row;
  float scale;
};
struct NsCall {
  int n_layers, steps, nesterov;
  float eps;
  const float* hparams;              // [count, 3] learning rate, momentum, weight decay; NULL: no momentum
  float coef[POP_NS_MAX_STEPS][3];
  float most;                        // singular values that start within [0, 1] stay below this in every step,
  float gain[POP_NS_MAX_STEPS + 1];  // and within gain[k] of what they started from in front of step k
  int segment;                       // steps taken in the space of X X^T before X itself is multiplied
  float q_most[POP_NS_MAX_STEPS];    // within which the steps of a segment up to step k multiply a singular value
  NsLayer layer[POP_MUON_MAX_LAYERS];
};
int64_t ns_most_workgroups(int64_t rows, int64_t cols);         // of one matrix, in units of 256 work items, in any launch
int64_t ns_workspace_bytes(int count, int rows, int cols);      // of one layer, a multiple of 256
hipError_t launch_ns(const NsCall& c, int dtype, void* ws, hipStream_t s);

}  // namespace pop
