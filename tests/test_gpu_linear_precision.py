"""Computed operands of linear attention for 16-bit arrays: weights of pairs, states and keys times their decay are taken to 24 bits, so that
sums which cancel leave what fp32 would."""
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from linear_common import BF16, F16, F32, OPERAND, OUT, UNIT, check, make, numpy_of, plan_of
from oracle import linear as L

pytestmark = pytest.mark.gpu
COLUMNS = 512


@pytest.fixture(autouse=True, scope="module")
def _built():
    ensure_built()


def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _near(got, want, size, dtype, units):
    """Within `units` of 2^-24 of the terms' magnitudes, then rounded to the type."""
    rel, least = OUT[dtype]
    off, tol = (got.double() - want).abs(), units * UNIT * size * (1 + rel) + rel * want.abs() + least
    assert bool((off <= tol).all()), (float((off / tol).max()), int((off > tol).sum()), off.numel())


def _ones(T, dtype, heads=COLUMNS):
    return torch.ones((1, 1, T, heads, 1), dtype=dtype, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_weights_of_pairs(dtype):
    """o_1 = lambda - what the type has of lambda.  Off by |z| * 1.25 units for exp2's argument (a constant to 2^-26, a product), two for exp2,
    two for the sum of two terms: under 8 of lambda + |v_1|."""
    z = -torch.rand((1, COLUMNS), generator=_gen(1), device="cuda")
    lam = torch.exp(z.double()).view(1, 1, COLUMNS, 1)
    one, v = _ones(2, dtype), _ones(2, dtype)
    v[:, :, 1] = -lam.to(dtype)
    plan = pp.LinearAttention(1, 1, 2, COLUMNS, 1, 1, dtype, scale=1.0)
    o, _ = plan.forward(one, one, v, z)
    assert bool((o[:, :, 0] == 1).all())
    _near(o[:, :, 1], lam + v[:, :, 1].double(), lam + v[:, :, 1].double().abs(), dtype, 8)
    # and from the end: dv_0 = k_0 (q_0 do_0 + lambda q_1 do_1)
    do = _ones(2, dtype)
    do[:, :, 0] = -lam.to(dtype)
    _, dk, dv, _ = plan.backward(one, one, one, do, z)
    for d in (dk, dv):
        _near(d[:, :, 0], lam + do[:, :, 0].double(), lam + do[:, :, 0].double().abs(), dtype, 8)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_states(dtype):
    """o_0 = S - what the type has of S, and each gradient's state alike: nothing but the sum is rounded, under 8 units of the terms."""
    one = _ones(1, dtype)
    S = 0.5 + 0.5 * torch.rand((1, 1, COLUMNS, 1, 1), generator=_gen(2), device="cuda")
    v = -S.view(1, 1, 1, COLUMNS, 1).to(dtype)
    want, size = S.double().view(v.shape) + v.double(), S.double().view(v.shape) + v.double().abs()
    plan = pp.LinearAttention(1, 1, 1, COLUMNS, 1, 1, dtype, scale=1.0)
    _near(plan.forward(one, one, v, state0=S)[0], want, size, dtype, 8)
    _near(plan.backward(one, one, v, one, state0=S)[0], want, size, dtype, 8)
    _, dk, dv, _ = plan.backward(one, one, one, v, dstate_last=S)
    for d in (dk, dv):
        _near(d, want, size, dtype, 8)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_states_in_front_of_segments(dtype):
    """One key at the front of 16 chunks, found again at their end: powers of lambda in products, one for the key's decay, one for each of up to 16
    chunks and 16 segments and one on the way out, are off by 5 units each at most (|n z| <= 1 in each): 34 * 5 = 170; few of them at once, and no chunk counts
    both in its segment and as one: 18 * 5 = 90."""
    T, H = 512, 64
    z = -torch.linspace(0.0002, 0.002, H, device="cuda").view(1, H)
    plan = pp.LinearAttention(1, 1, T, H, 1, 1, dtype, scale=1.0)
    lam = torch.exp(z.double() * (T - 1)).view(1, 1, H, 1)
    q = _ones(T, dtype, H)
    k, v = torch.zeros_like(q), torch.zeros_like(q)
    k[:, :, [0, -1]] = 1
    v[:, :, 0], v[:, :, -1] = 1, -lam.to(dtype)
    end = v[:, :, -1].double()
    _near(plan.forward(q, k, v, z)[0][:, :, -1], lam + end, lam + end.abs(), dtype, 90)
    # dq_{T-1} = S do; from the end q and do in the places of k and v, dv_0 = D k
    _near(plan.backward(q, k, v, q, z)[0][:, :, -1], lam + end, lam + end.abs(), dtype, 90)
    _, dk, dv, _ = plan.backward(k, q, q, v.flip(2), z)
    for d in (dk, dv):
        _near(d[:, :, 0], lam + end, lam + end.abs(), dtype, 90)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape", [(1, 2, 77, 1, 5, 128), (2, 1, 130, 1, 64, 64), (1, 2, 700, 2, 66, 30)])
def test_outputs_within_the_bound_of_32_bits(shape, dtype):
    """All that the oracle's bound for fp32 operands allows, and one rounding to the type."""
    c, do, dlast = make(shape, dtype, seed=3, reset=0.01, state0=True)
    given, plan = {k: numpy_of(x) for k, x in c.items()}, plan_of(shape, dtype)
    want, last, E = L.forward(**given, unit=UNIT, operand=OPERAND[F32])
    o, got_last = plan.forward(**c)
    check("o", o, want, E["o"], dtype)
    check("state_last", got_last, last, E["state_last"])
    want, E = L.backward(**given, do=numpy_of(do), dstate_last=numpy_of(dlast), unit=UNIT, operand=OPERAND[F32])
    for name, x in zip(("dq", "dk", "dv"), plan.backward(do=do, dstate_last=dlast, **c)):
        check(name, x, want[name], E[name], dtype)
