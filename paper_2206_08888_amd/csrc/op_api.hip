// C boundary of the operators (include/pop.h): argument checks on the host, then one launch wrapper.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include "operators.h"
#include "regions.h"

namespace pop {
namespace op {

constexpr int64_t kAlignment = 256;          // of a workspace
// a launch's work items per grid dimension stay below 2^32: one per column in a single step, up to eight over sequences
constexpr int64_t kMaxLanes = 1ll << 31, kMaxColumns = 1ll << 28;
constexpr int kMaxSteps = 1 << 22;           // steps and tiles are counted in ints, with room to spare; longer sequences go in pieces
constexpr int64_t kMaxWorkgroups = 1 << 21;  // of one layer's matrices

constexpr double kMostSingular = 8.0;

int64_t element_bytes(int32_t dtype) { return dtype == POP_F32 ? 4 : 2; }

int check_recurrence(const pop_recurrence_config* c) {
  if (!c) return fail_thread(POP_EINVAL, "config is NULL");
  if (c->P < 1 || c->batch < 1 || c->C < 1 || c->T < 0) return fail_thread(POP_EINVAL, "config: P, batch and C must be positive, T not negative");
  if (c->dtype != POP_F32 && c->dtype != POP_BF16 && c->dtype != POP_F16) return fail_thread(POP_EINVAL, "config: unknown dtype %d", c->dtype);
  if ((int64_t)c->P * c->batch >= kMaxLanes / c->C) return fail_thread(POP_EUNSUPPORTED, "P * batch * C must be below 2^31");
  if (c->T > kMaxSteps) return fail_thread(POP_EUNSUPPORTED, "T must be at most %d", kMaxSteps);
  return POP_OK;
}

int check_columns(const pop_recurrence_config* c) {
  if ((int64_t)c->P * c->batch * c->C > kMaxColumns) return fail_thread(POP_EUNSUPPORTED, "P * batch * C must be at most 2^28 but for single steps");
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

int check_apart(const Regions& r) {
  const char *one, *other;
  return r.clash(one, other) ? fail_thread(POP_EINVAL, "%s and %s overlap", one, other) : POP_OK;
}

void add_sequence(Regions& r, const pop_recurrence_config* c, const pop_sequence& s, const char* name, int64_t bytes, int64_t inner, bool written, int same = 0) {
  const int64_t n[3] = {c->P, c->batch, c->T}, stride[3] = {s.agent * bytes, s.row * bytes, s.step * bytes};
  r.add(name, s.data, inner * bytes, 3, n, stride, written, same);
}

void add_matrices(Regions& r, int64_t count, int64_t rows, int64_t cols, const pop_matrices& m, const char* name, int64_t bytes, bool written, int same = 0) {
  const int64_t n[2] = {count, rows}, stride[2] = {m.matrix * bytes, m.row * bytes};
  r.add(name, m.data, cols * bytes, 2, n, stride, written, same);
}

// NsCall::most, gain and q_most (segment is set).  p(s) = k0 s + k1 s^3 + k2 s^5 is largest at an end of the interval or where p' = 0, a quadratic
// in s^2; p(s) / s at an end or where its derivative in s^2 is 0.
void bounds_of(const pop_ns_config& c, NsCall& n) {
  double top = 1.0, gain = 1.0, in_segment = 1.0;
  n.most = 1.0f;
  for (int k = 0; k < c.steps; ++k) {
    n.gain[k] = (float)fmin(gain, 1e30);
    const double k0 = c.coef[k][0], k1 = c.coef[k][1], k2 = c.coef[k][2], end = top * top;
    const auto ratio = [&](double q) { return fabs(k0 + k1 * q + k2 * q * q); };             // q = s^2
    double next = ratio(end) * top, most = fmax(ratio(0.0), ratio(end));
    const auto turn = [&](double q) { if (q > 0.0 && q < end) next = fmax(next, ratio(q) * sqrt(q)); };
    const double d = 9 * k1 * k1 - 20 * k0 * k2;
    if (k2 != 0.0 && d >= 0.0) { turn((-3 * k1 + sqrt(d)) / (10 * k2)); turn((-3 * k1 - sqrt(d)) / (10 * k2)); }
    if (k2 == 0.0 && k1 != 0.0) turn(-k0 / (3 * k1));
    if (k2 != 0.0 && -k1 / (2 * k2) > 0.0 && -k1 / (2 * k2) < end) most = fmax(most, ratio(-k1 / (2 * k2)));
    top = next;
    gain *= most;
    in_segment = (k % n.segment == 0 ? 1.0 : in_segment) * most;
    n.q_most[k] = (float)fmin(in_segment, 1e30);
    n.most = (float)fmax(n.most, top);
    if (!(n.most <= kMostSingular)) return;
  }
  n.gain[c.steps] = (float)fmin(gain, 1e30);
}

// three: whether the results' type and the matrices' shape allow segments of three steps (k_orthogonalize.hip has the reasons)
int check_ns(const pop_ns_config* c, int32_t dtype, bool three, NsCall& n) {
  if (!c) return fail_thread(POP_EINVAL, "config is NULL");
  if (c->steps < 0 || c->steps > POP_NS_MAX_STEPS) return fail_thread(POP_EINVAL, "steps must be 0 .. %d", (int)POP_NS_MAX_STEPS);
  if (!(c->eps >= 1e-30f && c->eps <= 1e30f)) return fail_thread(POP_EINVAL, "eps must be within 1e-30 .. 1e30");
  if (dtype != POP_F32 && dtype != POP_BF16 && dtype != POP_F16) return fail_thread(POP_EINVAL, "unknown dtype %d", dtype);
  for (int k = 0; k < c->steps; ++k)
    for (float v : c->coef[k])
      if (!isfinite(v)) return fail_thread(POP_EINVAL, "coefficients of step %d are not finite", k);
  n = NsCall{};
  n.segment = 1;
  bounds_of(*c, n);
  if (three && n.gain[c->steps] <= kSegmentGain) {
    n.segment = 3;
    bounds_of(*c, n);
  }
  if (!(n.most <= kMostSingular)) return fail_thread(POP_EUNSUPPORTED, "the coefficients let singular values of at most 1 grow beyond %g", kMostSingular);
  n.steps = c->steps;
  n.eps = c->eps;
  for (int k = 0; k < c->steps; ++k)
    for (int i = 0; i < 3; ++i) n.coef[k][i] = c->coef[k][i];
  return POP_OK;
}

int check_shape(int64_t count, int64_t rows, int64_t cols) {
  if (count < 1 || rows < 1 || cols < 1) return fail_thread(POP_EINVAL, "a matrix count, rows or cols is not positive");
  if (rows > kNsMaxSide || cols > kNsMaxSide) return fail_thread(POP_EUNSUPPORTED, "rows and cols must be at most %d", kNsMaxSide);
  // a launch's work items, 256 for each workgroup of up to 8 layers, stay below 2^32 (a layer's workgroups are a multiple of 8)
  if ((count + 7) / 8 * 8 * ns_most_workgroups(rows, cols) >= kMaxWorkgroups)
    return fail_thread(POP_EUNSUPPORTED, "%lld matrices of %lld x %lld need 2^21 workgroups or more", (long long)count, (long long)rows, (long long)cols);
  return POP_OK;
}

int check_matrices(int64_t count, int64_t rows, int64_t cols, const pop_matrices& m, const char* name, bool output, int64_t bytes) {
  if (!m.data) return fail_thread(POP_EINVAL, "%s is NULL", name);
  if ((uintptr_t)m.data % bytes) return fail_thread(POP_EINVAL, "%s is not aligned to its type", name);
  const int64_t n[2] = {count, rows}, stride[2] = {m.matrix, m.row};
  if (output && !apart(cols, 2, n, stride)) return fail_thread(POP_EINVAL, "%s: its strides let elements overlap", name);
  return POP_OK;
}

int64_t muon_workspace(int32_t P, int32_t n_layers, const pop_muon_layer* layers) {
  if (n_layers < 1 || n_layers > POP_MUON_MAX_LAYERS) return fail_thread(POP_EINVAL, "n_layers must be 1 .. %d", (int)POP_MUON_MAX_LAYERS);
  if (!layers) return fail_thread(POP_EINVAL, "layers is NULL");
  int64_t sum = 0;
  for (int k = 0; k < n_layers; ++k) {
    const int rc = check_shape(P, layers[k].rows, layers[k].cols);
    if (rc != POP_OK) return rc;
    sum += ns_workspace_bytes(P, layers[k].rows, layers[k].cols);
  }
  return sum;
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

// The arrays of all three calls that only a direction of time reads, and those of x, g, y that this call has (y may be x or g in
// single steps: `same`).
Regions recurrence_regions(const pop_recurrence_config* c, const pop_recurrence_io* io, bool y, int same = 0) {
  Regions r;
  const int64_t e = element_bytes(c->dtype), rows = (int64_t)c->P * c->batch;
  if (c->T > 0) {
    add_sequence(r, c, io->x, "x", e, c->C, false, same);
    add_sequence(r, c, io->g, "g", e, c->C, false, same);
    if (y) add_sequence(r, c, io->y, "y", e, c->C, true, same);
    add_sequence(r, c, io->reset, "reset", 1, 1, false);
  }
  r.add("bias", io->bias, (int64_t)c->P * c->C * 4, false);
  r.add("lengths", io->lengths, rows * 4, false);
  return r;
}
enum { kStep = 1, kFirstAndLast = 2 };       // Region::same

}  // namespace op
}  // namespace pop

using namespace pop;
using namespace pop::op;

extern "C" {

int64_t pop_recurrence_workspace_bytes(const pop_recurrence_config* cfg) {
  const int rc = check_recurrence(cfg);
  return rc != POP_OK ? rc : (recur_workspace_floats(cfg->P, cfg->batch, cfg->T, cfg->C, element_bytes(cfg->dtype)) * 4 + kAlignment - 1) / kAlignment * kAlignment;
}

int64_t pop_recurrence_states_bytes(const pop_recurrence_config* cfg) {
  const int rc = check_recurrence(cfg);
  return rc != POP_OK ? rc : (int64_t)cfg->P * cfg->batch * recur_chunks(cfg->T) * cfg->C * 4;
}

int pop_recurrence_forward(const pop_recurrence_config* cfg, const pop_recurrence_io* io, void* workspace,
                           int64_t workspace_bytes, void* hip_stream) {
  RecurArgs a;
  int rc = recurrence_args(cfg, io, a);
  if (rc != POP_OK || (rc = check_columns(cfg)) != POP_OK) return rc;
  if (cfg->T > 0) {
    if ((rc = check_sequence(cfg, io->y, "y", true, element_bytes(cfg->dtype))) != POP_OK) return rc;
  }
  const int64_t need = pop_recurrence_workspace_bytes(cfg), rows = (int64_t)cfg->P * cfg->batch * cfg->C * 4;
  if ((rc = check_workspace(workspace, workspace_bytes, need)) != POP_OK) return rc;
  Regions r = recurrence_regions(cfg, io, true);
  r.add("h0", io->h0, rows, false, kFirstAndLast);
  r.add("h_last", io->h_last, rows, true, kFirstAndLast);
  r.add("states", io->states, rows * recur_chunks(cfg->T), true);
  r.add("workspace", workspace, need, true);
  if ((rc = check_apart(r)) != POP_OK) return rc;
  a.ws = (float*)workspace;
  return launched(launch_recur_forward(a, cfg->dtype, (hipStream_t)hip_stream));
}

int pop_recurrence_backward(const pop_recurrence_config* cfg, const pop_recurrence_io* io, const pop_recurrence_grads* grads,
                            void* workspace, int64_t workspace_bytes, void* hip_stream) {
  RecurArgs a;
  int rc = recurrence_args(cfg, io, a);
  if (rc != POP_OK || (rc = check_columns(cfg)) != POP_OK) return rc;
  if (!grads) return fail_thread(POP_EINVAL, "grads is NULL");
  if ((rc = check_floats(grads->dh_last, "dh_last", false)) != POP_OK || (rc = check_floats(grads->dh0, "dh0", false)) != POP_OK ||
      (rc = check_floats(grads->dbias, "dbias", false)) != POP_OK)
    return rc;
  if (cfg->T > 0) {
    const int64_t e = element_bytes(cfg->dtype);
    if ((rc = check_floats(io->states, "states", true)) != POP_OK || (rc = check_sequence(cfg, grads->dy, "dy", false, e)) != POP_OK ||
        (rc = check_sequence(cfg, grads->dx, "dx", true, e)) != POP_OK || (rc = check_sequence(cfg, grads->dg, "dg", true, e)) != POP_OK)
      return rc;
  }
  const int64_t need = pop_recurrence_workspace_bytes(cfg), rows = (int64_t)cfg->P * cfg->batch * cfg->C * 4;
  if ((rc = check_workspace(workspace, workspace_bytes, need)) != POP_OK) return rc;
  Regions r = recurrence_regions(cfg, io, false);
  if (cfg->T > 0) {
    const int64_t e = element_bytes(cfg->dtype);
    add_sequence(r, cfg, grads->dy, "dy", e, cfg->C, false);
    add_sequence(r, cfg, grads->dx, "dx", e, cfg->C, true);
    add_sequence(r, cfg, grads->dg, "dg", e, cfg->C, true);
    r.add("states", io->states, rows * recur_chunks(cfg->T), false);
  }
  r.add("dh_last", grads->dh_last, rows, false, kFirstAndLast);
  r.add("dh0", grads->dh0, rows, true, kFirstAndLast);
  r.add("dbias", grads->dbias, (int64_t)cfg->P * cfg->C * 4, true);
  r.add("workspace", workspace, need, true);
  if ((rc = check_apart(r)) != POP_OK) return rc;
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
  Regions r = recurrence_regions(cfg, io, true, kStep);
  r.add("slots", slots, (int64_t)cfg->P * cfg->batch * 4, false);
  r.add("state", state, (int64_t)cfg->P * n_slots * cfg->C * 4, true);
  if ((rc = check_apart(r)) != POP_OK) return rc;
  a.state = state; a.n_slots = n_slots; a.slots = slots;
  return launched(launch_recur_step(a, cfg->dtype, (hipStream_t)hip_stream));
}

int64_t pop_orthogonalize_workspace_bytes(int32_t count, int32_t rows, int32_t cols) {
  const int rc = check_shape(count, rows, cols);
  return rc != POP_OK ? rc : ns_workspace_bytes(count, rows, cols);
}

int pop_orthogonalize(const pop_ns_config* cfg, int32_t count, int32_t rows, int32_t cols, int32_t dtype, const pop_matrices* g,
                      const pop_matrices* out, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  NsCall n;
  const int64_t side = rows < cols ? rows : cols, other = rows < cols ? cols : rows;
  int rc = check_ns(cfg, dtype, dtype != POP_F32 && 2 * other >= 3 * side, n);
  if (rc != POP_OK || (rc = check_shape(count, rows, cols)) != POP_OK) return rc;
  if (!g || !out) return fail_thread(POP_EINVAL, "g or out is NULL");
  if ((rc = check_matrices(count, rows, cols, *g, "g", false, element_bytes(dtype))) != POP_OK ||
      (rc = check_matrices(count, rows, cols, *out, "out", true, element_bytes(dtype))) != POP_OK)
    return rc;
  const int64_t need = ns_workspace_bytes(count, rows, cols);
  if ((rc = check_workspace(workspace, workspace_bytes, need)) != POP_OK) return rc;
  Regions r;
  add_matrices(r, count, rows, cols, *g, "g", element_bytes(dtype), false, 1);
  add_matrices(r, count, rows, cols, *out, "out", element_bytes(dtype), true, 1);
  r.add("workspace", workspace, need, true);
  if ((rc = check_apart(r)) != POP_OK) return rc;
  n.n_layers = 1;
  NsLayer& l = n.layer[0];
  l.rows = rows; l.cols = cols; l.count = count;
  l.g = g->data; l.g_matrix = g->matrix; l.g_row = g->row;
  l.out = out->data; l.out_matrix = out->matrix; l.out_row = out->row;
  return launched(launch_ns(n, dtype, workspace, (hipStream_t)hip_stream));
}

int64_t pop_muon_workspace_bytes(int32_t P, int32_t n_layers, const pop_muon_layer* layers) { return muon_workspace(P, n_layers, layers); }

int pop_muon_step(const pop_ns_config* cfg, int32_t P, int32_t n_layers, const pop_muon_layer* layers, int32_t dtype, int32_t nesterov,
                  const pop_muon_hparams* hparams, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  NsCall n;
  int rc = check_ns(cfg, dtype, false, n);
  if (rc != POP_OK) return rc;
  const int64_t need = muon_workspace(P, n_layers, layers);
  if (need < 0) return (int)need;
  if ((rc = check_floats(hparams, "hparams", true)) != POP_OK) return rc;
  n.n_layers = n_layers;
  n.nesterov = nesterov != 0;
  n.hparams = (const float*)hparams;
  Regions r;
  r.add("hparams", hparams, (int64_t)P * sizeof(pop_muon_hparams), false);
  for (int k = 0; k < n_layers; ++k) {
    const pop_muon_layer& m = layers[k];
    if ((rc = check_matrices(P, m.rows, m.cols, m.grad, "grad", false, element_bytes(dtype))) != POP_OK ||
        (rc = check_matrices(P, m.rows, m.cols, m.momentum, "momentum", true, 4)) != POP_OK ||
        (rc = check_matrices(P, m.rows, m.cols, m.weight, "weight", true, 4)) != POP_OK)
      return rc;
    if (!isfinite(m.scale)) return fail_thread(POP_EINVAL, "layer %d: scale is not finite", k);
    NsLayer& l = n.layer[k];
    l.rows = m.rows; l.cols = m.cols; l.count = P; l.scale = m.scale;
    l.g = m.grad.data; l.g_matrix = m.grad.matrix; l.g_row = m.grad.row;
    l.momentum = (float*)m.momentum.data; l.m_matrix = m.momentum.matrix; l.m_row = m.momentum.row;
    l.weight = (float*)m.weight.data; l.w_matrix = m.weight.matrix; l.w_row = m.weight.row;
    add_matrices(r, P, m.rows, m.cols, m.grad, "a layer's grad", element_bytes(dtype), false);
    add_matrices(r, P, m.rows, m.cols, m.momentum, "a layer's momentum", 4, true);
    add_matrices(r, P, m.rows, m.cols, m.weight, "a layer's weight", 4, true);
  }
  if ((rc = check_workspace(workspace, workspace_bytes, need)) != POP_OK) return rc;
  r.add("workspace", workspace, need, true);
  if ((rc = check_apart(r)) != POP_OK) return rc;
  return launched(launch_ns(n, dtype, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
