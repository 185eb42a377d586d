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
  pop_sequence x, g, y, reset;       // step strides of single-step calls are set by the boundary
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
int64_t recur_workspace_floats(int64_t P, int64_t B, int64_t T, int64_t C);
hipError_t launch_recur_forward(const RecurArgs& a, int dtype, hipStream_t s);
hipError_t launch_recur_backward(const RecurArgs& a, int dtype, hipStream_t s);
hipError_t launch_recur_step(const RecurArgs& a, int dtype, hipStream_t s);

}  // namespace pop
