"""Operators for populations of recurrent agents on device tensors: the gated linear recurrence, linear attention with a decay
for each head, clipping of gradients by their norm, and the orthogonalised (Muon) update.  Argument marshalling for the calls
of include/pop.h of the same names; everything is computed in the HIP kernels of libpop.so, on PyTorch's current stream,
asynchronously.

Outputs and workspaces come from PyTorch's allocator, call by call, so calls may run on any stream and inside
torch.cuda.graph; tensors used on another stream than their own need the usual events and record_stream.

Autograd records none of this: backward passes are calls of their own.  Inputs that require gradients are refused while
gradients are recorded (pass them detached, or under torch.no_grad()); Muon, as optimisers do, updates weights outside of any
graph.  Tensors that are written in place raise their version, so that graphs which kept them notice.
"""
import ctypes as ct
import struct

import torch
from torch.autograd.graph import increment_version

from .binding import (  # noqa: F401
    CLIP_MAX_TENSORS, MUON_MAX_LAYERS, NS_COEF, NS_MAX_STEPS, POP_BF16, POP_F16, POP_F32, _check, load_library, make_ns_config,
    pop_gradient, pop_heads, pop_linear_config, pop_linear_grads, pop_linear_io, pop_matrices, pop_muon_layer, pop_ns_config,
    pop_recurrence_config, pop_recurrence_grads, pop_recurrence_io, pop_sequence,
)

DTYPE_CODES = {torch.float32: POP_F32, torch.bfloat16: POP_BF16, torch.float16: POP_F16}


def _dtype_code(dtype):
    if dtype not in DTYPE_CODES:
        raise ValueError("dtype must be torch.float32, torch.bfloat16 or torch.float16, not %s" % (dtype,))
    return DTYPE_CODES[dtype]


def _sizes(*sizes):
    """The boundary's numbers are of 32 bits, and ctypes cuts off what does not fit."""
    for v in sizes:
        if not -1 << 31 <= v < 1 << 31:
            raise ValueError("size %d does not fit in 32 bits" % v)


# current_stream(index).cuda_stream, where PyTorch has it without the object around it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


class _Operator:
    """Device and type checks, and the stream of a call.  Calls are short beside their launches, so the checks take the
    shortest way through what is right and find out what is wrong afterwards."""

    outside_graphs = False                               # whether tensors may require gradients

    def __init__(self, dtype, device):
        self.dtype, self.code = dtype, _dtype_code(dtype)
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("device must be a cuda device, not %s" % (device,))
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.index = self.device.index
        self.lib = load_library()

    def _tensor(self, t, name, shape, dtype=None, contiguous=True):
        dtype = dtype or self.dtype
        try:
            if (t.shape == shape and t.dtype is dtype and t.get_device() == self.index and (not contiguous or t.is_contiguous())
                    and (not t.requires_grad or self.outside_graphs or not torch.is_grad_enabled())):
                return t
        except AttributeError:
            pass
        if not isinstance(t, torch.Tensor) or t.device != self.device:
            raise ValueError("%s must be a tensor on %s" % (name, self.device))
        if t.dtype != dtype:
            raise ValueError("%s must be of type %s, not %s" % (name, dtype, t.dtype))
        if t.shape != shape:
            raise ValueError("%s must have shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
        if contiguous and not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
        raise ValueError("%s requires gradients, which are not recorded here: pass it detached or under torch.no_grad()" % name)

    def _pointer(self, t, name, shape, dtype=torch.float32):
        return None if t is None else self._tensor(t, name, shape, dtype).data_ptr()

    def _reset(self, reset, shape):
        if reset is None:
            return None, 0, 0, 0
        dtype = torch.bool if getattr(reset, "dtype", None) is torch.bool else torch.uint8
        s = self._tensor(reset, "reset", shape, dtype, contiguous=False).stride()
        return reset.data_ptr(), s[0], s[1], s[2] if len(s) == 3 else 0

    def _state_table(self, state, axes, slots):
        """The number of slots of a table with as many axes as the text `axes` names."""
        if not isinstance(state, torch.Tensor) or state.dim() != axes.count(",") + 1:
            raise ValueError("state must be a [%s] tensor" % axes)
        n_slots = state.shape[1]
        if n_slots >> 31:
            _sizes(n_slots)
        if slots is None and n_slots < self.batch:
            raise ValueError("state has %d rows for %d sequences and no slots are given" % (n_slots, self.batch))
        return n_slots

    def _empty(self, shape, dtype=None):
        return torch.empty(shape, dtype=dtype or self.dtype, device=self.device)

    def _call(self, fn, *args):
        """Enqueue on the current stream of this operator's device."""
        if torch.cuda.current_device() == self.index:
            rc = fn(*args, _raw_stream(self.index))
        else:
            with torch.cuda.device(self.device):
                rc = fn(*args, _raw_stream(self.index))
        if rc:
            _check(rc)


class Recurrence(_Operator):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a_t = sigmoid(g_t + bias), for P agents with `batch` sequences of up to T
    steps and C channels each; where `reset` is not zero the state in front of that step counts as zero.

    x, g and the gradients: [P, batch, T', C] of `dtype`, T' <= T, any strides with adjacent channels.  bias [P, C],
    h0, h_last, dh_last, dh0 [P, batch, C] are float32; reset [P, batch, T'] is uint8 or bool; lengths [P, batch] is
    int32: steps from a sequence's length on are not used, their outputs are zero."""

    def __init__(self, P, batch, T, C, dtype=torch.float32, device="cuda"):
        super().__init__(dtype, device)
        _sizes(P, batch, T, C)
        self.P, self.batch, self.T, self.C = P, batch, T, C
        self._rows, self._channels = (P, batch, C), (P, C)
        self._cfg = pop_recurrence_config(P, batch, T, C, self.code, 0)
        self._one = pop_recurrence_config(P, batch, 1, C, self.code, 0)
        self._one_ref = ct.byref(self._one)
        _check(self.lib.pop_recurrence_workspace_bytes(ct.byref(self._cfg)))

    def _sequence(self, t, name, shape):
        """The fields of a pop_sequence of [P, batch, T, C], or [P, batch, C] for single steps."""
        s = self._tensor(t, name, shape, contiguous=False).stride()
        if s[-1] != 1 and self.C > 1:
            raise ValueError("%s: its channels must be adjacent" % name)
        return t.data_ptr(), s[0], s[1], s[2] if len(s) == 4 else 0

    def _io(self, x, g, bias, h0, reset, lengths):
        T = x.shape[2] if x.dim() == 4 else -1
        if T < 0 or T > self.T:
            raise ValueError("x must have shape [%d, %d, up to %d, %d], not %s" % (self.P, self.batch, self.T, self.C, tuple(x.shape)))
        shape = (self.P, self.batch, T, self.C)
        io = pop_recurrence_io(self._sequence(x, "x", shape), self._sequence(g, "g", shape), (None, 0, 0, 0), self._reset(reset, shape[:3]),
                               self._pointer(bias, "bias", shape[::3]), self._pointer(h0, "h0", self._rows), None,
                               self._pointer(lengths, "lengths", shape[:2], torch.int32))
        return pop_recurrence_config(self.P, self.batch, T, self.C, self.code, 0), io, shape

    def _workspace(self, cfg):
        n = _check(self.lib.pop_recurrence_workspace_bytes(ct.byref(cfg)))
        return self._empty(n, torch.uint8), n

    def forward(self, x, g, bias=None, h0=None, reset=None, lengths=None, save=False):
        """(y, h_last); with save also the states that `backward` needs: (y, h_last, states)."""
        cfg, io, shape = self._io(x, g, bias, h0, reset, lengths)
        y, h_last = self._empty(shape), self._empty(self._rows, torch.float32)
        io.y, io.h_last = self._sequence(y, "y", shape), h_last.data_ptr()
        states = None
        if save:
            states = self._empty(_check(self.lib.pop_recurrence_states_bytes(ct.byref(cfg))) // 4, torch.float32)
            io.states = states.data_ptr()
        ws, n = self._workspace(cfg)
        self._call(self.lib.pop_recurrence_forward, ct.byref(cfg), ct.byref(io), ws.data_ptr(), n)
        return (y, h_last, states) if save else (y, h_last)

    def backward(self, states, x, g, dy, bias=None, reset=None, lengths=None, dh_last=None):
        """(dx, dg, dbias, dh0) of sum(y dy) + sum(h_last dh_last), from what `forward` was given and its states."""
        cfg, io, shape = self._io(x, g, bias, None, reset, lengths)
        n = _check(self.lib.pop_recurrence_states_bytes(ct.byref(cfg))) // 4
        io.states = self._pointer(states, "states", (n,))
        dx, dg = self._empty(shape), self._empty(shape)
        dbias, dh0 = self._empty(self._channels, torch.float32), self._empty(self._rows, torch.float32)
        grads = pop_recurrence_grads(self._sequence(dy, "dy", shape), self._sequence(dx, "dx", shape), self._sequence(dg, "dg", shape),
                                     self._pointer(dh_last, "dh_last", self._rows), dh0.data_ptr(), dbias.data_ptr())
        ws, n = self._workspace(cfg)
        self._call(self.lib.pop_recurrence_backward, ct.byref(cfg), ct.byref(io), ct.byref(grads), ws.data_ptr(), n)
        return dx, dg, dbias, dh0

    def step(self, x, g, state, bias=None, reset=None, slots=None):
        """One step of acting agents: x, g, y [P, batch, C]; state [P, n_slots, C] float32 is updated in place.  slots
        [P, batch] int32 names each row's state (none twice within an agent); a row whose slot is negative or not
        below n_slots is idle and gets zeros.  Without slots row b has state b."""
        shape = self._rows
        n_slots = self._state_table(state, "P, n_slots, C", slots)
        xs, gs = self._sequence(x, "x", shape), self._sequence(g, "g", shape)
        y = x.new_empty(shape)
        io = pop_recurrence_io(xs, gs, (y.data_ptr(), self.batch * self.C, self.C, 0), self._reset(reset, shape[:2]),
                               self._pointer(bias, "bias", self._channels))
        self._call(self.lib.pop_recurrence_step, self._one_ref, ct.byref(io), self._pointer(state, "state", (self.P, n_slots, self.C)),
                   n_slots, self._pointer(slots, "slots", shape[:2], torch.int32))
        increment_version(state)
        return y


class LinearAttention(_Operator):
    """A matrix for a memory: S_t = exp(log_decay) S_{t-1} + k_t v_t^T and o_t = scale S_t^T q_t, for P agents with `batch`
    sequences of up to T steps and `heads` heads each; where `reset` is not zero the state in front of that step counts as zero.

    q, k [P, batch, T', heads, key_dim], v, o [P, batch, T', heads, value_dim] and their gradients are of `dtype`, T' <= T, any
    strides with adjacent channels; both widths at most 128.  log_decay [P, heads] (at most 0; None: nothing decays) and the states
    state0, state_last, dstate_last, dstate0 [P, batch, heads, key_dim, value_dim] are float32; reset and lengths as in Recurrence.
    scale: by default key_dim ** -0.5; for float16 at most 2 ** 80."""

    def __init__(self, P, batch, T, heads, key_dim, value_dim, dtype=torch.float32, device="cuda", scale=None):
        super().__init__(dtype, device)
        _sizes(P, batch, T, heads, key_dim, value_dim)
        self.P, self.batch, self.T, self.heads, self.key_dim, self.value_dim = P, batch, T, heads, key_dim, value_dim
        self.scale = max(1, key_dim) ** -0.5 if scale is None else float(scale)
        self._decays, self._states = (P, heads), (P, batch, heads, key_dim, value_dim)
        _check(self.lib.pop_linear_forward_workspace_bytes(ct.byref(self._config(T))))
        self._one = self._config(1)
        self._one_ref = ct.byref(self._one)
        self._bytes = {}

    def _config(self, T):
        return pop_linear_config(self.P, self.batch, T, self.heads, self.key_dim, self.value_dim, self.code, self.scale)

    def _heads(self, t, name, shape):
        """The fields of a pop_heads of [P, batch, T, heads, width], or [P, batch, heads, width] for single steps."""
        s = self._tensor(t, name, shape, contiguous=False).stride()
        if s[-1] != 1 and shape[-1] > 1:
            raise ValueError("%s: its channels must be adjacent" % name)
        return (t.data_ptr(), s[0], s[1], s[2], s[3]) if len(s) == 5 else (t.data_ptr(), s[0], s[1], 0, s[2])

    def _io(self, q, k, v, log_decay, state0, reset, lengths):
        T = q.shape[2] if q.dim() == 5 else -1
        if T < 0 or T > self.T:
            raise ValueError("q must have shape [%d, %d, up to %d, %d, %d], not %s"
                             % (self.P, self.batch, self.T, self.heads, self.key_dim, tuple(q.shape)))
        keys, values = (self.P, self.batch, T, self.heads, self.key_dim), (self.P, self.batch, T, self.heads, self.value_dim)
        io = pop_linear_io(self._heads(q, "q", keys), self._heads(k, "k", keys), self._heads(v, "v", values), (None, 0, 0, 0, 0),
                           self._reset(reset, keys[:3]), self._pointer(log_decay, "log_decay", self._decays),
                           self._pointer(state0, "state0", self._states), None, self._pointer(lengths, "lengths", keys[:2], torch.int32))
        return self._config(T), io, keys, values

    def _workspace(self, sizes, cfg):
        n = self._bytes.get((sizes, cfg.T))
        if n is None:
            n = self._bytes[sizes, cfg.T] = _check(getattr(self.lib, sizes)(ct.byref(cfg)))
        return self._empty(n, torch.uint8), n

    def forward(self, q, k, v, log_decay=None, state0=None, reset=None, lengths=None):
        """(o, state_last)"""
        cfg, io, _, values = self._io(q, k, v, log_decay, state0, reset, lengths)
        o, last = self._empty(values), self._empty(self._states, torch.float32)
        io.o, io.state_last = self._heads(o, "o", values), last.data_ptr()
        ws, n = self._workspace("pop_linear_forward_workspace_bytes", cfg)
        self._call(self.lib.pop_linear_forward, ct.byref(cfg), ct.byref(io), ws.data_ptr(), n)
        return o, last

    def backward(self, q, k, v, do, log_decay=None, state0=None, reset=None, lengths=None, dstate_last=None):
        """(dq, dk, dv, dstate0) of sum(o do) + sum(state_last dstate_last), from what `forward` was given."""
        cfg, io, keys, values = self._io(q, k, v, log_decay, state0, reset, lengths)
        dq, dk, dv, dstate0 = self._empty(keys), self._empty(keys), self._empty(values), self._empty(self._states, torch.float32)
        grads = pop_linear_grads(self._heads(do, "do", values), self._heads(dq, "dq", keys), self._heads(dk, "dk", keys),
                                 self._heads(dv, "dv", values), self._pointer(dstate_last, "dstate_last", self._states), dstate0.data_ptr())
        ws, n = self._workspace("pop_linear_backward_workspace_bytes", cfg)
        self._call(self.lib.pop_linear_backward, ct.byref(cfg), ct.byref(io), ct.byref(grads), ws.data_ptr(), n)
        return dq, dk, dv, dstate0

    def step(self, q, k, v, state, log_decay=None, reset=None, slots=None):
        """One step of acting agents: q, k [P, batch, heads, key_dim], v, o [P, batch, heads, value_dim]; state [P, n_slots, heads,
        key_dim, value_dim] float32 is updated in place.  slots as in Recurrence.step."""
        n_slots = self._state_table(state, "P, n_slots, heads, key_dim, value_dim", slots)
        rows = (self.P, self.batch)
        keys, values = (*rows, self.heads, self.key_dim), (*rows, self.heads, self.value_dim)
        qs, ks, vs = self._heads(q, "q", keys), self._heads(k, "k", keys), self._heads(v, "v", values)
        o = v.new_empty(values)
        io = pop_linear_io(qs, ks, vs, (o.data_ptr(), self.batch * self.heads * self.value_dim, self.heads * self.value_dim, 0, self.value_dim),
                           self._reset(reset, rows), self._pointer(log_decay, "log_decay", self._decays))
        self._call(self.lib.pop_linear_step, self._one_ref, ct.byref(io), self._pointer(state, "state", (self.P, n_slots, *self._states[2:])),
                   n_slots, self._pointer(slots, "slots", rows, torch.int32))
        increment_version(state)
        return o


class _Stacks(_Operator):
    def _matrices(self, t, name, shape, dtype=None):
        t = self._tensor(t, name, shape, dtype, contiguous=False)
        s = t.stride()
        if s[2] != 1 and shape[2] > 1:
            raise ValueError("%s: its columns must be adjacent" % name)
        return pop_matrices(t.data_ptr(), s[0], s[1])


class Orthogonalizer(_Stacks):
    """orthogonalizer(g): Newton-Schulz products drive the singular values of every matrix of g [count, rows, cols]
    towards 1 (the products an orthogonalised optimiser takes its updates through).  Any strides with adjacent columns."""

    def __init__(self, count, rows, cols, dtype=torch.float32, device="cuda", steps=5, coef=NS_COEF, eps=1e-7):
        super().__init__(dtype, device)
        _sizes(count, rows, cols)
        self.shape = (count, rows, cols)
        self._ns = make_ns_config(steps, coef, eps)
        self._bytes = _check(self.lib.pop_orthogonalize_workspace_bytes(count, rows, cols))

    def __call__(self, g, out=None):
        """A new tensor, or `out` (which may be g)."""
        given, out = out, self._empty(self.shape) if out is None else out
        gm, om = self._matrices(g, "g", self.shape), self._matrices(out, "out", self.shape)
        ws = self._empty(self._bytes, torch.uint8)
        self._call(self.lib.pop_orthogonalize, ct.byref(self._ns), *self.shape, self.code, ct.byref(gm), ct.byref(om),
                   ws.data_ptr(), self._bytes)
        if given is not None:
            increment_version(given)
        return out


class Muon(_Stacks):
    """One optimiser step for the weight matrices of P agents, layer by layer [P, rows, cols]:

      M = mu M + G;  U = G + mu M (nesterov) or M;  W = (1 - lr wd) W - lr scale O,  O = U orthogonalised

    Weights and momenta are float32, gradients of `dtype`; any strides with adjacent columns.  shapes: (rows, cols) of
    each layer (at most 8); scales: a factor of each layer's update, by default sqrt(max(1, cols / rows)) (weights are
    [in, out])."""

    outside_graphs = True

    def __init__(self, P, shapes, dtype=torch.float32, device="cuda", scales=None, nesterov=True, steps=5, coef=NS_COEF, eps=1e-7):
        super().__init__(dtype, device)
        self.P, self.shapes, self.nesterov = P, [tuple(s) for s in shapes], nesterov
        _sizes(P, *(n for s in self.shapes for n in s))
        scales = [max(1.0, c / r) ** 0.5 for r, c in self.shapes] if scales is None else list(scales)
        if len(scales) != len(self.shapes):
            raise ValueError("%d scales for %d layers" % (len(scales), len(self.shapes)))
        self._ns = make_ns_config(steps, coef, eps)
        self._layers = (pop_muon_layer * max(1, len(self.shapes)))()
        for l, (r, c), f in zip(self._layers, self.shapes, scales):
            l.rows, l.cols, l.scale = r, c, f
        self._bytes = _check(self.lib.pop_muon_workspace_bytes(P, len(self.shapes), self._layers))

    def step(self, weights, momenta, grads, hparams):
        """weights, momenta (both updated in place), grads: one tensor per layer.  hparams: float32 tensor [P, 3] on the
        device, learning rate, momentum and weight decay of every agent."""
        if not len(weights) == len(momenta) == len(grads) == len(self.shapes):
            raise ValueError("weights, momenta and grads must have %d tensors each" % len(self.shapes))
        layers = (pop_muon_layer * len(self.shapes)).from_buffer_copy(self._layers)
        for l, (r, c), w, m, g in zip(layers, self.shapes, weights, momenta, grads):
            shape = (self.P, r, c)
            l.weight, l.momentum = self._matrices(w, "weight", shape, torch.float32), self._matrices(m, "momentum", shape, torch.float32)
            l.grad = self._matrices(g, "grad", shape)
        ws = self._empty(self._bytes, torch.uint8)
        self._call(self.lib.pop_muon_step, ct.byref(self._ns), self.P, len(self.shapes), layers, self.code, int(self.nesterov),
                   self._pointer(hparams, "hparams", (self.P, 3)), ws.data_ptr(), self._bytes)
        increment_version([*weights, *momenta])


class GradientClip(_Stacks):
    """clip(grads, max_norm): the norm of every agent's gradients over all tensors of the list, and the gradients scaled down where
    it is above the agent's limit:

      norm_i = sqrt(sum g^2);  out = g where norm_i + eps <= max_norm_i, else g max_norm_i / (norm_i + eps)

    shapes: of each tensor (at most 256) behind the agents' axis, e.g. (17, 256), (256,); tensors of three axes or fewer may have any
    strides with an adjacent last one, an agent's part of others lies in one piece.  dtype: one for all, or a list."""

    def __init__(self, P, shapes, dtype=torch.float32, device="cuda", eps=1e-6):
        dtypes = list(dtype) if isinstance(dtype, (list, tuple)) else [dtype] * len(shapes)
        super().__init__(dtypes[0] if dtypes else dtype, device)
        self.P, self.eps, self.shapes, self.dtypes = P, float(eps), [(P, *s) for s in shapes], dtypes
        if len(dtypes) != len(self.shapes):
            raise ValueError("%d types for %d tensors" % (len(dtypes), len(self.shapes)))
        self._layout = (pop_gradient * max(1, len(self.shapes)))()
        for g, shape, dt in zip(self._layout, self.shapes, dtypes):
            rows = 1
            for v in shape[1:-1]:
                rows *= v
            _sizes(*shape, rows)
            g.rows, g.cols, g.dtype = rows, shape[-1] if len(shape) > 1 else 1, _dtype_code(dt)
        self._bytes = _check(self.lib.pop_clip_workspace_bytes(P, len(self.shapes), self._layout))
        self._agents, self._call_layout = (P,), type(self._layout)
        self._words = [struct.unpack("2q", bytes(g)[:16]) for g in self._layout]
        self._strides = [(g.rows * g.cols, g.cols) for g in self._layout]      # of new tensors
        self._no_outs = [(0, 0, 0)] * len(self.shapes)
        self._pack = struct.Struct("%dq" % (8 * len(self.shapes))).pack

    def _list(self, tensors, name):
        """The fields of a pop_matrices for each of them."""
        if len(tensors) != len(self.shapes):
            raise ValueError("%s must have %d tensors, not %d" % (name, len(self.shapes), len(tensors)))
        fields = []
        for t, shape, dt in zip(tensors, self.shapes, self.dtypes):
            s = self._tensor(t, name, shape, dt, contiguous=False).stride()
            if len(s) <= 3:
                if len(s) > 1 and s[-1] != 1 and shape[-1] > 1:
                    raise ValueError("%s: its last axis must be adjacent" % name)
                fields.append((t.data_ptr(), s[0], s[1] if len(s) == 3 else 0))
            else:
                if not t[0].is_contiguous():
                    raise ValueError("%s: an agent's part of a tensor of %d axes must be contiguous" % (name, len(s)))
                fields.append((t.data_ptr(), s[0], shape[-1]))
        return fields

    def _run(self, grads, outs, max_norm):
        words = []                                       # the structures as words of 64 bits, the quickest way to fill them
        for layout, g, o in zip(self._words, self._list(grads, "grads"), outs):
            words += layout
            words += g
            words += o
        layout = self._call_layout.from_buffer_copy(self._pack(*words))
        norms, ws = self._empty(self._agents, torch.float32), self._empty(self._bytes, torch.uint8)
        self._call(self.lib.pop_clip_gradients, self.P, len(self.shapes), layout, self.eps, max_norm, norms.data_ptr(), ws.data_ptr(), self._bytes)
        return norms

    def __call__(self, grads, max_norm, out=None):
        """(clipped, norms): new tensors, or those of the list `out` (which may be grads, with the same strides).  max_norm: float32
        tensor [P] on the device.  norms [P]: float32, before clipping."""
        limits = self._tensor(max_norm, "max_norm", self._agents, torch.float32).data_ptr()
        if out is not None:
            norms = self._run(grads, self._list(out, "out"), limits)
            increment_version(list(out))
            return out, norms
        out = [torch.empty(s, dtype=dt, device=self.device) for s, dt in zip(self.shapes, self.dtypes)]
        return out, self._run(grads, [(t.data_ptr(), *s) for t, s in zip(out, self._strides)], limits)

    def norms(self, grads):
        """The norms alone: float32 [P]."""
        return self._run(grads, self._no_outs, None)
