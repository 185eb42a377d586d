"""Linear attention and clipping, CPU-only: structures as in the header, refusals before any GPU work."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2206_08888_amd as pp
from test_operators_boundary import ADDRESS, ROOT, lib, ops, test_structures_match_the_header as _structure  # noqa: F401

WS = 1 << 30
BIG = 1 << 40


@pytest.mark.parametrize("name", ["pop_linear_config", "pop_heads", "pop_linear_io", "pop_linear_grads", "pop_gradient"])
def test_structures(lib, tmp_path, name):  # noqa: F811
    _structure(lib, tmp_path, name)


def _config(**kw):
    base = dict(P=2, batch=3, T=20, heads=2, key_dim=4, value_dim=5, dtype=pp.POP_F32, scale=0.5)
    return ops.pop_linear_config(**dict(base, **kw))


def _heads(width, at, T=20, batch=3, heads=2):
    return ops.pop_heads(at * ADDRESS, batch * T * heads * width, T * heads * width, heads * width, width)


def _io(T=20, **kw):
    io = ops.pop_linear_io()
    io.q, io.k, io.v, io.o = _heads(4, 1, T), _heads(4, 2, T), _heads(5, 3, T), _heads(5, 4, T)
    for k, v in kw.items():
        setattr(io, k, v)
    return io


def _grads(**kw):
    g = ops.pop_linear_grads()
    g.d_o, g.dq, g.dk, g.dv = _heads(5, 5), _heads(4, 6), _heads(4, 7), _heads(5, 8)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def _forward(lib, io, cfg=None, ws=WS, size=BIG):  # noqa: F811
    return lib.pop_linear_forward(C.byref(cfg or _config()), C.byref(io) if io else None, ws, size, None)


def _backward(lib, io, grads, cfg=None, ws=WS, size=BIG):  # noqa: F811
    return lib.pop_linear_backward(C.byref(cfg or _config()), C.byref(io), C.byref(grads) if grads else None, ws, size, None)


@pytest.mark.parametrize("kw, code", [
    (dict(P=0), pp.POP_EINVAL), (dict(batch=0), pp.POP_EINVAL), (dict(heads=0), pp.POP_EINVAL), (dict(key_dim=0), pp.POP_EINVAL), (dict(value_dim=-1), pp.POP_EINVAL),
    (dict(T=-1), pp.POP_EINVAL), (dict(dtype=3), pp.POP_EINVAL), (dict(scale=float("nan")), pp.POP_EINVAL), (dict(scale=float("inf")), pp.POP_EINVAL),
    (dict(key_dim=129), pp.POP_EUNSUPPORTED), (dict(value_dim=129), pp.POP_EUNSUPPORTED), (dict(T=(1 << 22) + 1), pp.POP_EUNSUPPORTED),
    (dict(P=1 << 12, batch=1 << 11, heads=2), pp.POP_EUNSUPPORTED), (dict(P=1 << 30, batch=1 << 30, heads=1 << 30), pp.POP_EUNSUPPORTED)])
def test_configs(lib, kw, code):  # noqa: F811
    cfg = _config(**kw)
    assert lib.pop_linear_forward_workspace_bytes(C.byref(cfg)) == code
    assert lib.pop_linear_backward_workspace_bytes(C.byref(cfg)) == code
    assert pp.pop_last_error(None) != ""
    assert _forward(lib, _io(), cfg) == code and _backward(lib, _io(), _grads(), cfg) == code
    assert lib.pop_linear_step(C.byref(cfg), C.byref(_io()), 9 * ADDRESS, 3, None, None) == code


def test_sizes(lib):  # noqa: F811
    for kw in (dict(), dict(T=0), dict(T=1 << 22, P=1, batch=1, key_dim=128, value_dim=128), dict(P=1 << 20, batch=1)):
        for size in (lib.pop_linear_forward_workspace_bytes, lib.pop_linear_backward_workspace_bytes):
            n = size(C.byref(_config(**kw)))
            assert n >= 0 and n % 256 == 0, kw


@pytest.mark.parametrize("kw", [
    dict(q=ops.pop_heads(None, 0, 0, 0, 0)), dict(k=ops.pop_heads(ADDRESS + 2, 480, 160, 8, 4)), dict(v=ops.pop_heads(None, 0, 0, 0, 0)), dict(o=ops.pop_heads(None, 0, 0, 0, 0)),
    dict(o=ops.pop_heads(4 * ADDRESS, 600, 200, 10, 0)),                    # heads on top of each other
    dict(o=ops.pop_heads(4 * ADDRESS, 600, 200, 10, 4)),                    # and closer than their channels
    dict(o=ops.pop_heads(4 * ADDRESS, 600, 0, 10, 5)), dict(log_decay=ADDRESS + 1), dict(state0=ADDRESS + 2), dict(state_last=ADDRESS + 3), dict(lengths=ADDRESS + 2)])
def test_forward_refuses(lib, kw):  # noqa: F811
    assert _forward(lib, _io(**kw)) == pp.POP_EINVAL
    assert pp.pop_last_error(None) != ""


def test_workspaces(lib):  # noqa: F811
    long = _config(P=1, batch=1, heads=1, T=20000)
    io = _io()
    for n in ("q", "k", "v", "o"):
        setattr(io, n, ops.pop_heads(getattr(io, n).data, 0, 0, 5, 0))
    for size, call in ((lib.pop_linear_forward_workspace_bytes, lambda *a: _forward(lib, io, long, *a)),
                       (lib.pop_linear_backward_workspace_bytes, lambda *a: _backward(lib, io, _long_grads(), long, *a))):
        need = size(C.byref(long))
        if need == 0:
            continue
        assert call(None, need) == pp.POP_EINVAL and call(WS + 128, need) == pp.POP_EINVAL and call(WS, need - 1) == pp.POP_ENOMEM
    assert _forward(lib, None) == pp.POP_EINVAL and _backward(lib, _io(), None) == pp.POP_EINVAL
    assert lib.pop_linear_forward(None, C.byref(io), WS, BIG, None) == pp.POP_EINVAL


def _long_grads():
    g = ops.pop_linear_grads()
    for i, n in enumerate(("d_o", "dq", "dk", "dv")):
        setattr(g, n, ops.pop_heads((5 + i) * ADDRESS, 0, 0, 5, 0))
    return g


@pytest.mark.parametrize("kw", [
    dict(d_o=ops.pop_heads(None, 0, 0, 0, 0)), dict(dq=ops.pop_heads(None, 0, 0, 0, 0)), dict(dk=ops.pop_heads(7 * ADDRESS, 480, 160, 8, 0)),
    dict(dv=ops.pop_heads(8 * ADDRESS + 1, 600, 200, 10, 5)), dict(dstate_last=ADDRESS + 2), dict(dstate0=ADDRESS + 2)])
def test_backward_refuses(lib, kw):  # noqa: F811
    assert _backward(lib, _io(), _grads(**kw)) == pp.POP_EINVAL


def _overlaps(rc, *names):
    assert rc == pp.POP_EINVAL
    message = pp.pop_last_error(None)
    assert "overlap" in message and all(n in message for n in names), message


@pytest.mark.parametrize("kw, names", [
    (dict(o=_heads(5, 1)), ("q", "o")), (dict(o=ops.pop_heads(4 * ADDRESS - 4, 600, 200, 10, 5), v=ops.pop_heads(4 * ADDRESS, 600, 200, 10, 5)), ("v", "o")),
    (dict(state_last=4 * ADDRESS + 100), ("o", "state_last")), (dict(state0=9 * ADDRESS, state_last=9 * ADDRESS + 4), ("state0", "state_last")),
    (dict(log_decay=4 * ADDRESS), ("o", "log_decay")), (dict(lengths=4 * ADDRESS + 8), ("o", "lengths")), (dict(reset=ops.pop_sequence(4 * ADDRESS, 60, 20, 1)), ("o", "reset"))])
def test_forward_overlaps(lib, kw, names):  # noqa: F811
    _overlaps(_forward(lib, _io(**kw)), *names)


@pytest.mark.parametrize("kw, names", [
    (dict(dq=_heads(4, 1)), ("q", "dq")), (dict(dk=_heads(4, 6)), ("dq", "dk")), (dict(dv=_heads(5, 5)), ("d_o", "dv")),
    (dict(dstate_last=9 * ADDRESS, dstate0=9 * ADDRESS), ("dstate_last", "dstate0")), (dict(dstate0=8 * ADDRESS), ("dv", "dstate0"))])
def test_backward_overlaps(lib, kw, names):  # noqa: F811
    _overlaps(_backward(lib, _io(), _grads(**kw)), *names)


def test_interleaved_outputs_pass_the_checks(lib):  # noqa: F811
    """dq, dk and dv as the parts of one array [P, batch, T, 2, 13]: refused only for what does reach into one of them."""
    wide = lambda off: ops.pop_heads(16 * ADDRESS + 4 * off, 3 * 20 * 26, 20 * 26, 26, 13)
    io = _io()
    _overlaps(_backward(lib, io, _grads(dq=wide(0), dk=wide(4), dv=wide(8), dstate0=16 * ADDRESS)), "dq", "dstate0")
    _overlaps(_backward(lib, io, _grads(dq=wide(0), dk=wide(4), dv=wide(8), dstate0=16 * ADDRESS + 4 * 26 * 20 * 6 - 4)), "dv", "dstate0")
    _overlaps(_backward(lib, io, _grads(dq=wide(0), dk=wide(3), dv=wide(8))), "dq", "dk")


@pytest.mark.parametrize("kw", [dict(state0=ADDRESS), dict(state_last=ADDRESS), dict(lengths=ADDRESS)])
def test_step_refuses(lib, kw):  # noqa: F811
    one = _config(T=1)
    call = lambda cfg, io, state, n, slots=None: lib.pop_linear_step(C.byref(cfg), C.byref(io) if io else None, state, n, slots, None)
    assert call(one, _io(1, **kw), 9 * ADDRESS, 3) == pp.POP_EINVAL
    assert call(_config(), _io(), 9 * ADDRESS, 3) == pp.POP_EINVAL          # T is not 1
    assert call(one, None, 9 * ADDRESS, 3) == pp.POP_EINVAL
    assert call(one, _io(1), None, 3) == pp.POP_EINVAL and call(one, _io(1), 9 * ADDRESS + 2, 3) == pp.POP_EINVAL
    assert call(one, _io(1), 9 * ADDRESS, 0) == pp.POP_EINVAL
    assert call(one, _io(1), 9 * ADDRESS, 3, ADDRESS + 1) == pp.POP_EINVAL
    _overlaps(call(one, _io(1), 4 * ADDRESS, 3), "o", "state")
    _overlaps(call(one, _io(1), 9 * ADDRESS, 3, 9 * ADDRESS), "slots", "state")
    _overlaps(call(one, _io(1, o=_heads(5, 3, 1)), 9 * ADDRESS, 3), "v", "o")
    big = _config(T=1, P=1 << 20, batch=1, heads=8, key_dim=128, value_dim=128)
    io = ops.pop_linear_io(*(_heads(128, k << 14, 1, 1, 8) for k in (1, 2, 3, 4)))
    assert call(big, io, 9 * ADDRESS, (1 << 31) - 1) == pp.POP_EUNSUPPORTED


def _clip(lib, n=2, P=2, eps=1e-6, limits=50 * ADDRESS, norms=51 * ADDRESS, ws=WS, size=BIG, none=False, **kw):  # noqa: F811
    grads = (ops.pop_gradient * max(n, 2))()
    for k, g in enumerate(grads):
        g.rows, g.cols, g.dtype = 5, 6, pp.POP_F32
        g.grad, g.out = ops.pop_matrices((1 + 2 * (k % 20)) * ADDRESS, 30, 6), ops.pop_matrices((2 + 2 * (k % 20)) * ADDRESS, 30, 6)
    for k, v in kw.items():
        setattr(grads[0], k, v)
    return lib.pop_clip_gradients(P, n, None if none else grads, eps, limits, norms, ws, size, None)


@pytest.mark.parametrize("kw, code", [
    (dict(P=0), pp.POP_EINVAL), (dict(n=0), pp.POP_EINVAL), (dict(n=257), pp.POP_EINVAL), (dict(none=True), pp.POP_EINVAL), (dict(rows=0), pp.POP_EINVAL),
    (dict(cols=0), pp.POP_EINVAL), (dict(dtype=5), pp.POP_EINVAL), (dict(eps=-1.0), pp.POP_EINVAL), (dict(eps=float("nan")), pp.POP_EINVAL), (dict(eps=float("inf")), pp.POP_EINVAL),
    (dict(limits=ADDRESS + 1), pp.POP_EINVAL), (dict(norms=ADDRESS + 1), pp.POP_EINVAL), (dict(limits=None, norms=None), pp.POP_EINVAL),
    (dict(grad=ops.pop_matrices(None, 30, 6)), pp.POP_EINVAL), (dict(out=ops.pop_matrices(None, 30, 6)), pp.POP_EINVAL), (dict(grad=ops.pop_matrices(ADDRESS + 2, 30, 6)), pp.POP_EINVAL),
    (dict(out=ops.pop_matrices(2 * ADDRESS, 0, 6)), pp.POP_EINVAL), (dict(out=ops.pop_matrices(2 * ADDRESS, 30, 5)), pp.POP_EINVAL),
    (dict(ws=None), pp.POP_EINVAL), (dict(ws=WS + 8), pp.POP_EINVAL), (dict(size=10), pp.POP_ENOMEM),
    (dict(rows=1 << 21, cols=1 << 21), pp.POP_EUNSUPPORTED), (dict(P=1 << 24), pp.POP_EUNSUPPORTED), (dict(P=1 << 14, cols=1 << 23, rows=1), pp.POP_EUNSUPPORTED)])
def test_clip_refuses(lib, kw, code):  # noqa: F811
    assert _clip(lib, **kw) == code
    assert pp.pop_last_error(None) != ""


@pytest.mark.parametrize("kw, names", [
    (dict(out=ops.pop_matrices(ADDRESS + 4, 30, 6)), ("a grad", "an out")), (dict(out=ops.pop_matrices(3 * ADDRESS, 30, 6)), ("a grad", "an out")),
    (dict(out=ops.pop_matrices(4 * ADDRESS + 4 * 59, 30, 6)), ("an out",)), (dict(out=ops.pop_matrices(ADDRESS, 60, 6)), ("a grad", "an out")),
    (dict(limits=2 * ADDRESS), ("an out", "max_norm")), (dict(norms=ADDRESS), ("a grad", "norms")), (dict(limits=51 * ADDRESS), ("max_norm", "norms")),
    (dict(norms=WS), ("norms", "workspace")), (dict(n=21), ("an out",))])
def test_clip_overlaps(lib, kw, names):  # noqa: F811
    _overlaps(_clip(lib, **kw), *names)


def test_meeting_regions_with_four_axes(tmp_path):
    """Regions of four axes against all of their bytes, and many at once against each pair."""
    exe = tmp_path / "many_regions_check"
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2206_08888_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "many_regions_check.cpp"), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and "bad 0" in out.stdout, out.stdout[-2000:]
