"""Cases of linear attention for the GPU tests: inputs in several memory layouts, and outputs held against the oracle in 64 bits, element
by element within the bound that it propagates."""
import numpy as np
import torch

import paper_2206_08888_amd as pp
from oracle import linear as L

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
OUT = {F32: (0.0, 0.0), BF16: (2.0 ** -8, 2.0 ** -133), F16: (2.0 ** -11, 2.0 ** -24)}   # half a unit, smallest value
UNIT = 2.0 ** -24
# what lies between an operand of a matrix product and the value it stands for: two parts of 8 bits each for outputs of 16 bits, three for fp32
# ones, states among them
OPERAND = {F32: 2.0 ** -23, BF16: 2.0 ** -16, F16: 2.0 ** -16}


def numpy_of(t):
    return None if t is None else t.detach().double().cpu().numpy()


def check(name, got, want, bound, dtype=F32):
    got, (rel, least) = numpy_of(got), OUT[dtype]
    assert got.shape == want.shape, name
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), (name, np.argwhere(fine != np.isfinite(got))[:3].tolist())
    with np.errstate(all="ignore"):
        tol = bound * (1 + rel) + rel * np.abs(want) + least + 1e-37
        bad = fine & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), bad.size, np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], tol[bad][:3])


def array(shape, dtype, gen, layout="plain", scale=1.0):
    """[P, B, T, H, D]; what lies between the elements is NaN."""
    P, B, T, H, D = shape
    v = (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)
    if layout == "time_major":
        return v.permute(2, 0, 1, 3, 4).contiguous().permute(1, 2, 0, 3, 4)
    if layout == "head_major":
        return v.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
    if layout == "packed":                               # the second part of a wider row, at an odd offset
        wide = torch.full((P, B, T, 2 * H * D + 3), float("nan"), dtype=dtype, device="cuda")
        part = wide[..., H * D + 3:].unflatten(-1, (H, D))
        part.copy_(v)
        return part
    if layout == "padded":                               # rows of whole 16 bytes, apart
        wide = torch.full((P, B, T, H, D + (-D) % 8 + 8), float("nan"), dtype=dtype, device="cuda")
        wide[..., :D] = v
        return wide[..., :D]
    if layout == "broadcast":                            # all heads and sequences share one
        return v[:, :1, :, :1].expand(shape)
    return v


def make(shape, dtype, seed=0, layout="plain", reset=0.0, ragged=False, state0=False, decay=(0.002, 0.3)):
    """(arguments of forward, do, dstate_last)"""
    P, B, T, H, K, V = shape
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c = {name: array((P, B, T, H, D), dtype, gen, layout) for name, D in (("q", K), ("k", K), ("v", V))}
    lo, hi = decay
    c["log_decay"] = -(lo + (hi - lo) * torch.rand((P, H), generator=gen, device="cuda"))
    c["reset"] = torch.rand((P, B, T), generator=gen, device="cuda") < reset if reset else None
    c["lengths"] = None
    if ragged:
        c["lengths"] = torch.randint(0, T + 1, (P, B), generator=gen, device="cuda", dtype=torch.int32)
        c["lengths"].view(-1)[0] = 0
        c["lengths"].view(-1)[-1] = T
    c["state0"] = torch.randn((P, B, H, K, V), generator=gen, device="cuda") if state0 else None
    do = array((P, B, T, H, V), dtype, gen, layout, 0.5)
    return c, do, torch.randn((P, B, H, K, V), generator=gen, device="cuda") if state0 else None


def plan_of(shape, dtype, **kw):
    return pp.LinearAttention(*shape, dtype, **kw)


def check_forward(shape, dtype, c, got=None, scale=None):
    o, last = plan_of(shape, dtype, scale=scale).forward(**c) if got is None else got
    given = {k: numpy_of(x) for k, x in c.items()}
    want, want_last, E = L.forward(**given, scale=scale, unit=UNIT, operand=OPERAND[dtype])
    check("o", o, want, E["o"], dtype)
    if dtype != F32:
        E = L.forward(**given, scale=scale, unit=UNIT, operand=OPERAND[F32])[2]
    check("state_last", last, want_last, E["state_last"])


def check_backward(shape, dtype, c, do, dlast, got=None, scale=None):
    got = plan_of(shape, dtype, scale=scale).backward(do=do, dstate_last=dlast, **c) if got is None else got
    given = dict({k: numpy_of(x) for k, x in c.items()}, do=numpy_of(do), dstate_last=numpy_of(dlast), scale=scale, unit=UNIT)
    want, E = L.backward(**given, operand=OPERAND[dtype])
    if dtype != F32:
        E = dict(E, dstate0=L.backward(**given, operand=OPERAND[F32])[1]["dstate0"])
    for name, x in zip(("dq", "dk", "dv", "dstate0"), got):
        check(name, x, want[name], E[name], F32 if name == "dstate0" else dtype)
