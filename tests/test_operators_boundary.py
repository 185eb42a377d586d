"""Operators, CPU-only: structures as in the header, refusals before any GPU work."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2206_08888_amd as pp
from paper_2206_08888_amd import operators as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pp.lib_path()):
        from paper_2206_08888_amd import build
        build.build()
    return pp.load_library()


STRUCTS = ("pop_recurrence_config", "pop_sequence", "pop_recurrence_io", "pop_recurrence_grads")


@pytest.mark.parametrize("name", STRUCTS)
def test_structures_match_the_header(lib, tmp_path, name):
    struct = getattr(ops, name)
    fields = [f for f, _ in struct._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "pop.h"\nint main(void) { printf("%%zu", sizeof(%s)); %s return 0; }\n'
                   % (name, " ".join('printf(" %%zu", offsetof(%s, %s));' % (name, f) for f in fields)))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(struct)] + [getattr(struct, f).offset for f in fields]


def _config(**kw):
    base = dict(P=2, batch=3, T=200, C=5, dtype=pp.POP_F32, reserved_=0)
    return ops.pop_recurrence_config(**dict(base, **kw))


ADDRESS = 1 << 20                                        # never read: the calls under test refuse first


def _sequence(C_=5, T=200, batch=3, at=ADDRESS):
    return ops.pop_sequence(at, batch * T * C_, T * C_, C_)


def _io(**kw):
    io = ops.pop_recurrence_io()
    io.x, io.g, io.y = _sequence(), _sequence(at=2 * ADDRESS), _sequence(at=3 * ADDRESS)
    for k, v in kw.items():
        setattr(io, k, v)
    return io


def _grads(**kw):
    g = ops.pop_recurrence_grads()
    g.dy, g.dx, g.dg = _sequence(at=4 * ADDRESS), _sequence(at=5 * ADDRESS), _sequence(at=6 * ADDRESS)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


@pytest.mark.parametrize("kw, code", [
    (dict(P=0), pp.POP_EINVAL), (dict(batch=0), pp.POP_EINVAL), (dict(C=0), pp.POP_EINVAL), (dict(T=-1), pp.POP_EINVAL),
    (dict(dtype=3), pp.POP_EINVAL), (dict(P=1 << 15, batch=1 << 15, C=2), pp.POP_EUNSUPPORTED), (dict(T=(1 << 22) + 1), pp.POP_EUNSUPPORTED)])
def test_recurrence_configs(lib, kw, code):
    cfg = _config(**kw)
    assert lib.pop_recurrence_workspace_bytes(C.byref(cfg)) == code
    assert lib.pop_recurrence_states_bytes(C.byref(cfg)) == code
    assert pp.pop_last_error(None) != ""
    assert lib.pop_recurrence_forward(C.byref(cfg), C.byref(_io()), ADDRESS, 1 << 40, None) == code


def test_recurrence_sizes(lib):
    cfg = _config()
    assert lib.pop_recurrence_states_bytes(C.byref(cfg)) == 2 * 3 * 2 * 5 * 4     # two chunks of 128 steps
    assert lib.pop_recurrence_workspace_bytes(C.byref(cfg)) % 256 == 0
    assert lib.pop_recurrence_states_bytes(C.byref(_config(T=0))) == 0


@pytest.mark.parametrize("kw", [
    dict(x=ops.pop_sequence(None, 0, 0, 0)), dict(g=_sequence(at=ADDRESS + 2)), dict(y=ops.pop_sequence(None, 0, 0, 0)),
    dict(y=ops.pop_sequence(3 * ADDRESS, 3000, 1000, 0)),               # a broadcast output
    dict(y=ops.pop_sequence(3 * ADDRESS, 3000, 4, 1000)),               # rows closer than their channels
    dict(y=ops.pop_sequence(3 * ADDRESS, 2000, 1000, 5)),               # an agent's rows reach into the next agent
    dict(y=_sequence()), dict(y=_sequence(at=2 * ADDRESS)), dict(bias=ADDRESS + 1), dict(h0=ADDRESS + 2),
    dict(h_last=ADDRESS + 3), dict(states=ADDRESS + 1), dict(lengths=ADDRESS + 2)])
def test_recurrence_forward_refuses(lib, kw):
    cfg = _config()
    assert lib.pop_recurrence_forward(C.byref(cfg), C.byref(_io(**kw)), ADDRESS, 1 << 40, None) == pp.POP_EINVAL
    assert pp.pop_last_error(None) != ""


def test_recurrence_workspaces_are_checked(lib):
    cfg, io = _config(), _io()
    need = lib.pop_recurrence_workspace_bytes(C.byref(cfg))
    assert lib.pop_recurrence_forward(C.byref(cfg), C.byref(io), None, need, None) == pp.POP_EINVAL
    assert lib.pop_recurrence_forward(C.byref(cfg), C.byref(io), ADDRESS + 128, need, None) == pp.POP_EINVAL
    assert lib.pop_recurrence_forward(C.byref(cfg), C.byref(io), ADDRESS, need - 1, None) == pp.POP_ENOMEM
    assert lib.pop_recurrence_forward(None, C.byref(io), ADDRESS, need, None) == pp.POP_EINVAL
    assert lib.pop_recurrence_forward(C.byref(cfg), None, ADDRESS, need, None) == pp.POP_EINVAL


@pytest.mark.parametrize("io_kw, grads_kw", [
    (dict(), dict()),                                                   # no states
    (dict(states=8 * ADDRESS), dict(dy=ops.pop_sequence(None, 0, 0, 0))),
    (dict(states=8 * ADDRESS), dict(dx=ops.pop_sequence(5 * ADDRESS, 0, 1000, 5))),
    (dict(states=8 * ADDRESS), dict(dg=_sequence(at=5 * ADDRESS))),
    (dict(states=8 * ADDRESS), dict(dx=_sequence())),
    (dict(states=8 * ADDRESS), dict(dg=_sequence(at=4 * ADDRESS))),
    (dict(states=8 * ADDRESS), dict(dh0=ADDRESS + 2)),
    (dict(states=8 * ADDRESS), dict(dbias=ADDRESS + 2)),
    (dict(states=8 * ADDRESS), dict(dh_last=ADDRESS + 2))])
def test_recurrence_backward_refuses(lib, io_kw, grads_kw):
    cfg = _config()
    io, grads = _io(**io_kw), _grads(**grads_kw)
    assert lib.pop_recurrence_backward(C.byref(cfg), C.byref(io), C.byref(grads), ADDRESS, 1 << 40, None) == pp.POP_EINVAL
    assert lib.pop_recurrence_backward(C.byref(cfg), C.byref(io), None, ADDRESS, 1 << 40, None) == pp.POP_EINVAL


@pytest.mark.parametrize("kw", [dict(h0=ADDRESS), dict(h_last=ADDRESS), dict(lengths=ADDRESS), dict(states=ADDRESS)])
def test_recurrence_step_refuses(lib, kw):
    one = _config(T=1)
    call = lambda cfg, io, state, n: lib.pop_recurrence_step(C.byref(cfg), C.byref(io), state, n, None, None)
    assert call(one, _io(**kw), ADDRESS, 3) == pp.POP_EINVAL
    assert call(_config(), _io(), ADDRESS, 3) == pp.POP_EINVAL          # T is not 1
    assert call(one, _io(), None, 3) == pp.POP_EINVAL
    assert call(one, _io(), ADDRESS + 2, 3) == pp.POP_EINVAL
    assert call(one, _io(), ADDRESS, 0) == pp.POP_EINVAL


@pytest.mark.parametrize("name", ["pop_ns_config", "pop_matrices", "pop_muon_layer"])
def test_structures_of_orthogonalised_updates_match_the_header(lib, tmp_path, name):
    test_structures_match_the_header(lib, tmp_path, name)


def _orthogonalize(lib, cfg=None, count=2, rows=5, cols=6, dtype=pp.POP_F32, g=(ADDRESS, 30, 6), out=(2 * ADDRESS, 30, 6),
                   ws=3 * ADDRESS, size=1 << 40):
    ref = lambda s: None if s is None else C.byref(ops.pop_matrices(*s))
    return lib.pop_orthogonalize(C.byref(cfg or pp.make_ns_config()), count, rows, cols, dtype, ref(g), ref(out), ws, size, None)


def _ns(**kw):
    cfg = pp.make_ns_config()
    for k, v in kw.items():
        setattr(cfg, k, v)
    return cfg


@pytest.mark.parametrize("kw, code", [
    (dict(count=0), pp.POP_EINVAL), (dict(rows=0), pp.POP_EINVAL), (dict(cols=-1), pp.POP_EINVAL), (dict(dtype=7), pp.POP_EINVAL),
    (dict(rows=16385), pp.POP_EUNSUPPORTED), (dict(cols=16385), pp.POP_EUNSUPPORTED), (dict(count=1 << 20), pp.POP_EUNSUPPORTED),
    (dict(g=None), pp.POP_EINVAL), (dict(out=None), pp.POP_EINVAL), (dict(g=(None, 30, 6)), pp.POP_EINVAL),
    (dict(g=(ADDRESS + 2, 30, 6)), pp.POP_EINVAL), (dict(out=(ADDRESS, 30, 6), g=(ADDRESS, 60, 6)), pp.POP_EINVAL),
    (dict(out=(2 * ADDRESS, 0, 6)), pp.POP_EINVAL), (dict(out=(2 * ADDRESS, 30, 5)), pp.POP_EINVAL), (dict(out=(2 * ADDRESS, 6, 6)), pp.POP_EINVAL),
    (dict(ws=None), pp.POP_EINVAL), (dict(ws=ADDRESS + 64), pp.POP_EINVAL), (dict(size=100), pp.POP_ENOMEM),
    (dict(cfg=_ns(steps=-1)), pp.POP_EINVAL), (dict(cfg=_ns(steps=17)), pp.POP_EINVAL), (dict(cfg=_ns(eps=0.0)), pp.POP_EINVAL),
    (dict(cfg=_ns(eps=float("nan"))), pp.POP_EINVAL)])
def test_orthogonalize_refuses(lib, kw, code):
    assert _orthogonalize(lib, **kw) == code
    assert pp.pop_last_error(None) != ""


@pytest.mark.parametrize("coef, code", [((float("nan"), 0, 0), pp.POP_EINVAL), ((9.0, 0.0, 0.0), pp.POP_EUNSUPPORTED),
                                        ((3.0, 0.0, 0.0), pp.POP_EUNSUPPORTED), ((1.5, 0.5, 0.0), pp.POP_EUNSUPPORTED),
                                        ((1.0, 30.0, -31.0), pp.POP_EUNSUPPORTED), ((1e30, 1e30, 1e30), pp.POP_EUNSUPPORTED)])
def test_coefficients_that_let_singular_values_grow_are_refused(lib, coef, code):
    """(1, 30, -31): 0 and 1 stay, what lies between grows to 8.3 and beyond."""
    assert _orthogonalize(lib, cfg=pp.make_ns_config(5, coef)) == code


def test_muon_refuses(lib):
    def call(P=2, n=1, dtype=pp.POP_F32, hp=5 * ADDRESS, ws=4 * ADDRESS, size=1 << 40, none=False, **kw):
        layers = (ops.pop_muon_layer * 9)()
        for l in layers:
            l.rows, l.cols, l.scale = 5, 6, 1.0
            l.grad, l.momentum, l.weight = (ops.pop_matrices(k * ADDRESS, 30, 6) for k in (1, 2, 3))
        for k, v in kw.items():
            setattr(layers[0], k, v)
        return lib.pop_muon_step(C.byref(pp.make_ns_config()), P, n, None if none else layers, dtype, 1, hp, ws, size, None)

    for kw in (dict(P=0), dict(n=0), dict(n=9), dict(none=True), dict(dtype=-1), dict(hp=None), dict(hp=ADDRESS + 1), dict(ws=None), dict(rows=0),
               dict(scale=float("inf")), dict(weight=ops.pop_matrices(2 * ADDRESS, 30, 6)), dict(grad=ops.pop_matrices(3 * ADDRESS, 30, 6)),
               dict(momentum=ops.pop_matrices(None, 30, 6)), dict(weight=ops.pop_matrices(3 * ADDRESS, 0, 6)),
               dict(grad=ops.pop_matrices(ADDRESS + 1, 30, 6))):
        assert call(**kw) == pp.POP_EINVAL, kw
    assert call(size=100) == pp.POP_ENOMEM
    assert call(rows=20000) == pp.POP_EUNSUPPORTED


def test_more_columns_than_a_grid_takes(lib):
    cfg, io = _config(P=1 << 14, batch=1 << 14, C=2), _io(states=8 * ADDRESS)
    assert lib.pop_recurrence_forward(C.byref(cfg), C.byref(io), ADDRESS, 1 << 60, None) == pp.POP_EUNSUPPORTED
    assert "2^28" in pp.pop_last_error(None)
    assert lib.pop_recurrence_backward(C.byref(cfg), C.byref(io), C.byref(_grads()), ADDRESS, 1 << 60, None) == pp.POP_EUNSUPPORTED
