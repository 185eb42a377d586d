"""Arrays that share memory, CPU-only: outputs over inputs, each other or the workspace are refused before any GPU work.  (Layouts
that reach into each other and keep apart, and results written over an input where that is allowed: test_gpu_operator_aliases.py
and test_gpu_operator_outputs.py.)"""
import ctypes as C
import os
import subprocess

import pytest

import paper_2206_08888_amd as pp
from test_operators_boundary import ADDRESS, ROOT, _config, _grads, _io, _orthogonalize, _sequence, lib, ops  # noqa: F401

WS = 1 << 30
N = 2 * 3 * 200 * 5 * 4                                  # bytes of a sequence


def test_meeting_regions(tmp_path):
    exe = tmp_path / "regions_check"
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2206_08888_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "regions_check.cpp"), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and "bad 0" in out.stdout, out.stdout[-2000:]


def _refused(rc, *names):
    assert rc == pp.POP_EINVAL
    message = pp.pop_last_error(None)
    assert "overlap" in message and all(n in message for n in names), message


@pytest.mark.parametrize("kw, names", [
    (dict(y=_sequence(at=ADDRESS + 20)), ("x", "y")),                   # a step further
    (dict(y=_sequence(at=2 * ADDRESS - N + 4)), ("g", "y")),            # its last element
    (dict(y=ops.pop_sequence(ADDRESS + 16, 6000, 2000, 10)), ("x", "y")),
    (dict(h_last=3 * ADDRESS + 400), ("y", "h_last")), (dict(h_last=ADDRESS), ("x", "h_last")),
    (dict(h0=4 * ADDRESS, h_last=4 * ADDRESS + 4), ("h0", "h_last")),
    (dict(bias=4 * ADDRESS, states=4 * ADDRESS + 36), ("bias", "states")),
    (dict(lengths=3 * ADDRESS + N - 4), ("lengths", "y")),
    (dict(reset=ops.pop_sequence(3 * ADDRESS - 1199, 600, 200, 1)), ("reset", "y")),
    (dict(h0=WS), ("h0", "workspace")), (dict(y=_sequence(at=WS - 4)), ("y", "workspace"))])
def test_forward(lib, kw, names):  # noqa: F811
    _refused(lib.pop_recurrence_forward(C.byref(_config()), C.byref(_io(**kw)), WS, 1 << 40, None), *names)


@pytest.mark.parametrize("kw, names", [
    (dict(dx=_sequence(at=ADDRESS + 4)), ("x", "dx")), (dict(dg=_sequence(at=5 * ADDRESS + 8)), ("dx", "dg")),
    (dict(dg=_sequence(at=4 * ADDRESS + 4000)), ("dy", "dg")), (dict(dbias=8 * ADDRESS), ("states", "dbias")),
    (dict(dh_last=9 * ADDRESS, dh0=9 * ADDRESS + 4), ("dh_last", "dh0")), (dict(dh0=5 * ADDRESS), ("dx", "dh0")),
    (dict(dh0=9 * ADDRESS, dbias=9 * ADDRESS), ("dh0", "dbias")), (dict(dx=_sequence(at=WS)), ("dx", "workspace"))])
def test_backward(lib, kw, names):  # noqa: F811
    io = _io(states=8 * ADDRESS)
    _refused(lib.pop_recurrence_backward(C.byref(_config()), C.byref(io), C.byref(_grads(**kw)), WS, 1 << 40, None), *names)


@pytest.mark.parametrize("kw, state, slots, names", [
    (dict(y=_sequence(T=1, at=ADDRESS + 4)), 9 * ADDRESS, None, ("x", "y")),
    (dict(y=ops.pop_sequence(ADDRESS, 20, 40, 0)), 9 * ADDRESS, None, ("x", "y")),          # x's place, other strides
    (dict(), ADDRESS, None, ("x", "state")), (dict(), 3 * ADDRESS + 116, None, ("y", "state")),
    (dict(), 9 * ADDRESS, 9 * ADDRESS + 7 * 20 * 2 - 4, ("slots", "state")), (dict(bias=9 * ADDRESS), 9 * ADDRESS, None, ("bias", "state"))])
def test_step(lib, kw, state, slots, names):  # noqa: F811
    io = _io(**dict(dict(x=_sequence(T=1), g=_sequence(T=1, at=2 * ADDRESS), y=_sequence(T=1, at=3 * ADDRESS)), **kw))
    _refused(lib.pop_recurrence_step(C.byref(_config(T=1)), C.byref(io), state, 7, slots, None), *names)


@pytest.mark.parametrize("kw, names", [(dict(out=(ADDRESS + 4, 30, 6)), ("g", "out")), (dict(out=(ADDRESS + 24, 30, 6)), ("g", "out")),
                                       (dict(out=(ADDRESS, 60, 6)), ("g", "out")), (dict(g=(WS + 64, 30, 6), ws=WS), ("g", "workspace"))])
def test_orthogonalize(lib, kw, names):  # noqa: F811
    _refused(_orthogonalize(lib, **kw), *names)


@pytest.mark.parametrize("at, names", [((1, 2, 3, 4, 5, 3), ("weight",)), ((1, 2, 3, 4, 2, 6), ("momentum",)), ((1, 2, 3, 3, 5, 6), ("grad", "weight")),
                                       ((1, 2, 3, 4, 5, 8), ("weight", "workspace")), ((1, 2, 9, 4, 5, 6), ("hparams", "weight"))])
def test_muon_layers(lib, at, names):  # noqa: F811
    layers = (ops.pop_muon_layer * 2)()
    for l, a in zip(layers, (at[:3], at[3:])):
        l.rows, l.cols, l.scale = 5, 6, 1.0
        l.grad, l.momentum, l.weight = (ops.pop_matrices(k * ADDRESS, 30, 6) for k in a)
    _refused(lib.pop_muon_step(C.byref(pp.make_ns_config()), 2, 2, layers, pp.POP_F32, 1, 9 * ADDRESS, 8 * ADDRESS, 1 << 40, None), *names)
