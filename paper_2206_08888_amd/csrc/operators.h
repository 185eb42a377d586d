// Operators for populations of recurrent agents: what the boundary (op_api.hip) hands to the launch wrappers of
// k_recurrence.hip and k_orthogonalize.hip.
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
