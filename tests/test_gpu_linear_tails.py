"""Activations of a projection where their results are far below 1 but not yet below what bf16 holds."""
import pytest
import torch

from tests.rows_common import Linear, act64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,lo,hi", [("silu", -105.0, -80.0), ("gelu_tanh", -11.0, -9.0), ("gelu", -14.0, -12.0),
                                       ("silu", -1.0, 1.0), ("gelu_tanh", -1.0, 1.0)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M", [10, 300, 2600])
def test_tails(act, lo, hi, gated, M):
    """x w^T = z exactly. An exponent of up to 150 is off by 4 roundings (150 x 2^-22 = 2^-14.8 of the result), a sigmoid
    of 2^-133 has 16 bits left (2^-17): 2^-14 with the fit and the reciprocal; the result's half step, 2^-8; numbers below
    fp32's normal ones (2^-126) may count as zero. Gated, the other factor is 1."""
    x = Linear("bf16", M, 8, 260, act=act, gated=gated)
    for t in (x.x, x.w) + ((x.w_up,) if gated else ()):
        t.zero_()
    x.x[:, 0] = torch.linspace(lo, hi, M, device="cuda").to(torch.bfloat16)
    x.x[:, 1] = 1.0
    x.w[:, 0] = 1.0
    if gated:
        x.w_up[:, 1] = 1.0
    x.call(x.workspace())
    z = x.x[:, :1].double()
    want = act64(z, act)
    tol = (2.0 ** -8 + 2.0 ** -14) * want.abs() + 2.0 ** -126
    off = (x.y.double() - want).abs() / tol
    worst = int(off.amax(1).argmax())
    assert bool((off <= 1).all()), f"z = {float(z[worst])}: {float(x.y[worst, 0])} for {float(want[worst])}"
