"""Operators for populations of recurrent agents on device tensors: the gated linear recurrence and the orthogonalised
(Muon) update.  Argument marshalling for the calls of include/pop.h of the same names; everything is computed in the
HIP kernels of libpop.so, on PyTorch's current stream, asynchronously.

Outputs and workspaces come from PyTorch's allocator, call by call, so calls may run on any stream and inside
torch.cuda.graph; tensors used on another stream than their own need the usual events and record_stream.

Autograd records none of this: backward passes are calls of their own.  Inputs that require gradients are refused while
gradients are recorded (pass them detached, or under torch.no_grad()); Muon, as optimisers do, updates weights outside of any
graph.  Tensors that are written in place raise their version, so that graphs which kept them notice.
"""
import ctypes as ct

import torch
from torch.autograd.graph import increment_version

from .binding import (  # noqa: F401
    MUON_MAX_LAYERS, NS_COEF, NS_MAX_STEPS, POP_BF16, POP_F16, POP_F32, _check, load_library, make_ns_config, pop_matrices,
    pop_muon_layer, pop_ns_config,
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

    def _reset(self, reset, shape):
        if reset is None:
            return None, 0, 0, 0
        dtype = torch.bool if getattr(reset, "dtype", None) is torch.bool else torch.uint8
        s = self._tensor(reset, "reset", shape, dtype, contiguous=False).stride()
        return reset.data_ptr(), s[0], s[1], s[2] if len(s) == 3 else 0

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
        if not isinstance(state, torch.Tensor) or state.dim() != 3:
            raise ValueError("state must be a [P, n_slots, C] tensor")
        n_slots = state.shape[1]
        if n_slots >> 31:
            _sizes(n_slots)
        if slots is None and n_slots < self.batch:
            raise ValueError("state has %d rows for %d sequences and no slots are given" % (n_slots, self.batch))
        xs, gs = self._sequence(x, "x", shape), self._sequence(g, "g", shape)
        y = x.new_empty(shape)
        io = pop_recurrence_io(xs, gs, (y.data_ptr(), self.batch * self.C, self.C, 0), self._reset(reset, shape[:2]),
                               self._pointer(bias, "bias", self._channels))
        self._call(self.lib.pop_recurrence_step, self._one_ref, ct.byref(io), self._pointer(state, "state", (self.P, n_slots, self.C)),
                   n_slots, self._pointer(slots, "slots", shape[:2], torch.int32))
        increment_version(state)
        return y


class _NewtonSchulz(_Operator):
    def _matrices(self, t, name, shape, dtype=None):
        t = self._tensor(t, name, shape, dtype, contiguous=False)
        s = t.stride()
        if s[2] != 1 and shape[2] > 1:
            raise ValueError("%s: its columns must be adjacent" % name)
        return pop_matrices(t.data_ptr(), s[0], s[1])


class Orthogonalizer(_NewtonSchulz):
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


class Muon(_NewtonSchulz):
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
