"""vt_linear and vt_linear_gated in the forms that tests/linear_plans.py lists, against float64, element by element."""
import pytest

from tests.linear_plans import FORMS
from tests.rows_common import MARK, Linear

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ws():
    return Linear("f16", 1, 8, 8).workspace()


@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,K,N,pad", FORMS)
def test_forms(ws, type, gated, M, K, N, pad):
    """The product alone, and with activation, bias and residual; equal calls give equal bits."""
    for more in (dict(), dict(act="gelu_tanh", bias=True, residual=True)):
        x = Linear(type, M, K, N, gated=gated, pad=pad, seed=M + K + N, **more)
        x.call(ws)
        x.check()
        first = x.y.clone()
        x.y.fill_(MARK)
        x.call(ws)
        assert bool((x.y == first).all()), "equal calls, other bits"
