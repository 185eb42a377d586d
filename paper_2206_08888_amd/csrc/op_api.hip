// C boundary of the operators (include/pop.h): argument checks on the host, then one launch wrapper.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include "operators.h"

namespace pop {
namespace op {

constexpr int64_t kAlignment = 256;          // of a workspace
constexpr int64_t kMaxLanes = 1ll << 31;     // a launch's work items per grid dimension stay below 2^32
constexpr int kMaxSteps = 1 << 22;           // chunks of a sequence are a grid dimension of at most 65,535

int64_t element_bytes(int32_t dtype) { return dtype == POP_F32 ? 4 : 2; }

int check_recurrence(const pop_recurrence_config* c) {
  if (!c) return fail_thread(POP_EINVAL, "config is NULL");
  if (c->P < 1 || c->batch < 1 || c->C < 1 || c->T < 0) return fail_thread(POP_EINVAL, "config: P, batch and C must be positive, T not negative");
  if (c->dtype != POP_F32 && c->dtype != POP_BF16 && c->dtype != POP_F16) return fail_thread(POP_EINVAL, "config: unknown dtype %d", c->dtype);
  if ((int64_t)c->P * c->batch >= kMaxLanes / c->C) return fail_thread(POP_EUNSUPPORTED, "P * batch * C must be below 2^31");
  if (c->T > kMaxSteps) return fail_thread(POP_EUNSUPPORTED, "T must be at most %d", kMaxSteps);
  return POP_OK;
}

int check_floats(const void* p, const char* name, bool needed) {
  if (!p && needed) return fail_thread(POP_EINVAL, "%s is NULL", name);
  if ((uintptr_t)p % 4) return fail_thread(POP_EINVAL, "%s is not aligned to its type", name);
  return POP_OK;
}

// Whether an array of n[i] blocks at stride[i] with `inner` adjacent elements surely has no element twice.
bool apart(int64_t inner, int axes, const int64_t* n, const int64_t* stride) {
  int64_t extent = inner;
  bool done[3] = {false, false, false};
  for (int k = 0; k < axes; ++k) {
    int next = -1;
    int64_t least = 0;
    for (int i = 0; i < axes; ++i) {
      const int64_t d = stride[i] < 0 ? -stride[i] : stride[i];
      if (!done[i] && (next < 0 || d < least)) { next = i; least = d; }
    }
    done[next] = true;
    if (n[next] < 2) continue;
    if (least < extent) return false;
    extent += least * (n[next] - 1);
  }
  return true;
}

int check_sequence(const pop_recurrence_config* c, const pop_sequence& s, const char* name, bool output, int64_t bytes) {
  if (!s.data) return fail_thread(POP_EINVAL, "%s is NULL", name);
  if ((uintptr_t)s.data % bytes) return fail_thread(POP_EINVAL, "%s is not aligned to its type", name);
  const int64_t n[3] = {c->P, c->batch, c->T}, stride[3] = {s.agent, s.row, s.step};
  if (output && !apart(c->C, 3, n, stride)) return fail_thread(POP_EINVAL, "%s: its strides let elements overlap", name);
  return POP_OK;
}

int check_workspace(void* p, int64_t have, int64_t need) {
  if (need == 0) return POP_OK;
  if (!p) return fail_thread(POP_EINVAL, "workspace is NULL");
  if ((uintptr_t)p % kAlignment) return fail_thread(POP_EINVAL, "workspace must be 256-byte aligned");
  if (have < need) return fail_thread(POP_ENOMEM, "workspace has %lld bytes, %lld needed", (long long)have, (long long)need);
  return POP_OK;
}

int launched(hipError_t e) { return e == hipSuccess ? POP_OK : fail_thread(POP_EHIP, "kernel launch: %s", hipGetErrorString(e)); }

// The parts of the arguments that all three calls share, checked.
int recurrence_args(const pop_recurrence_config* c, const pop_recurrence_io* io, RecurArgs& a) {
  int rc = check_recurrence(c);
  if (rc != POP_OK) return rc;
  if (!io) return fail_thread(POP_EINVAL, "io is NULL");
  a = RecurArgs{};
  a.P = c->P; a.B = c->batch; a.T = c->T; a.C = c->C;
  a.x = io->x; a.g = io->g; a.y = io->y; a.reset = io->reset;
  a.bias = io->bias; a.h0 = io->h0; a.lengths = io->lengths; a.h_last = io->h_last; a.states = io->states;
  if ((rc = check_floats(io->bias, "bias", false)) != POP_OK || (rc = check_floats(io->h0, "h0", false)) != POP_OK ||
      (rc = check_floats(io->h_last, "h_last", false)) != POP_OK || (rc = check_floats(io->states, "states", false)) != POP_OK ||
      (rc = check_floats(io->lengths, "lengths", false)) != POP_OK)
    return rc;
  if (c->T == 0) return POP_OK;
  const int64_t e = element_bytes(c->dtype);
  if ((rc = check_sequence(c, io->x, "x", false, e)) != POP_OK || (rc = check_sequence(c, io->g, "g", false, e)) != POP_OK) return rc;
  return POP_OK;
}

}  // namespace op
}  // namespace pop

using namespace pop;
using namespace pop::op;

extern "C" {

int64_t pop_recurrence_workspace_bytes(const pop_recurrence_config* cfg) {
  const int rc = check_recurrence(cfg);
  return rc != POP_OK ? rc : (recur_workspace_floats(cfg->P, cfg->batch, cfg->T, cfg->C) * 4 + kAlignment - 1) / kAlignment * kAlignment;
}

int64_t pop_recurrence_states_bytes(const pop_recurrence_config* cfg) {
  const int rc = check_recurrence(cfg);
  return rc != POP_OK ? rc : (int64_t)cfg->P * cfg->batch * recur_chunks(cfg->T) * cfg->C * 4;
}

int pop_recurrence_forward(const pop_recurrence_config* cfg, const pop_recurrence_io* io, void* workspace,
                           int64_t workspace_bytes, void* hip_stream) {
  RecurArgs a;
  int rc = recurrence_args(cfg, io, a);
  if (rc != POP_OK) return rc;
  if (cfg->T > 0) {
    if ((rc = check_sequence(cfg, io->y, "y", true, element_bytes(cfg->dtype))) != POP_OK) return rc;
    if (io->y.data == io->x.data || io->y.data == io->g.data) return fail_thread(POP_EINVAL, "y must not overlap x or g");
  }
  if ((rc = check_workspace(workspace, workspace_bytes, pop_recurrence_workspace_bytes(cfg))) != POP_OK) return rc;
  a.ws = (float*)workspace;
  return launched(launch_recur_forward(a, cfg->dtype, (hipStream_t)hip_stream));
}

int pop_recurrence_backward(const pop_recurrence_config* cfg, const pop_recurrence_io* io, const pop_recurrence_grads* grads,
                            void* workspace, int64_t workspace_bytes, void* hip_stream) {
  RecurArgs a;
  int rc = recurrence_args(cfg, io, a);
  if (rc != POP_OK) return rc;
  if (!grads) return fail_thread(POP_EINVAL, "grads is NULL");
  if ((rc = check_floats(grads->dh_last, "dh_last", false)) != POP_OK || (rc = check_floats(grads->dh0, "dh0", false)) != POP_OK ||
      (rc = check_floats(grads->dbias, "dbias", false)) != POP_OK)
    return rc;
  if (cfg->T > 0) {
    const int64_t e = element_bytes(cfg->dtype);
    if ((rc = check_floats(io->states, "states", true)) != POP_OK || (rc = check_sequence(cfg, grads->dy, "dy", false, e)) != POP_OK ||
        (rc = check_sequence(cfg, grads->dx, "dx", true, e)) != POP_OK || (rc = check_sequence(cfg, grads->dg, "dg", true, e)) != POP_OK)
      return rc;
    const void* outs[2] = {grads->dx.data, grads->dg.data};
    for (const void* o : outs)
      if (o == io->x.data || o == io->g.data || o == grads->dy.data) return fail_thread(POP_EINVAL, "dx and dg must not overlap x, g or dy");
    if (outs[0] == outs[1]) return fail_thread(POP_EINVAL, "dx and dg must not overlap");
  }
  if ((rc = check_workspace(workspace, workspace_bytes, pop_recurrence_workspace_bytes(cfg))) != POP_OK) return rc;
  a.dy = grads->dy; a.dx = grads->dx; a.dg = grads->dg;
  a.dh_last = grads->dh_last; a.dh0 = grads->dh0; a.dbias = grads->dbias;
  a.ws = (float*)workspace;
  return launched(launch_recur_backward(a, cfg->dtype, (hipStream_t)hip_stream));
}

int pop_recurrence_step(const pop_recurrence_config* cfg, const pop_recurrence_io* io, float* state, int32_t n_slots,
                        const int32_t* slots, void* hip_stream) {
  RecurArgs a;
  int rc = recurrence_args(cfg, io, a);
  if (rc != POP_OK) return rc;
  if (cfg->T != 1) return fail_thread(POP_EINVAL, "T must be 1 for a single step");
  if (io->h0 || io->h_last || io->lengths || io->states) return fail_thread(POP_EINVAL, "h0, h_last, lengths and states must be NULL for a single step");
  if ((rc = check_sequence(cfg, io->y, "y", true, element_bytes(cfg->dtype))) != POP_OK ||
      (rc = check_floats(state, "state", true)) != POP_OK || (rc = check_floats(slots, "slots", false)) != POP_OK)
    return rc;
  if (n_slots < 1) return fail_thread(POP_EINVAL, "n_slots must be positive");
  a.state = state; a.n_slots = n_slots; a.slots = slots;
  return launched(launch_recur_step(a, cfg->dtype, (hipStream_t)hip_stream));
}

}  // extern "C"
