"""How many digits the delta rule's fp32 arithmetic keeps, where a result shows them: sums that cancel."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from mixer_helpers import DELTA, UNITS          # noqa: E402
from oracle import mixers as om                 # noqa: E402
from token_helpers import TYPES, Gen, host      # noqa: E402


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("Dk", [24, 64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_sums_that_cancel(mb, dtype, Dk, states):
    """Results of a 16-bit type that are small next to their terms: what the products lost is not below their rounding.  The bound
    is that of the fp32 products, DELTA roundings of the results' size, with the half step of the small result itself."""
    B, L, H, Dv = 8, 64, 8, 128
    T, g = TYPES[dtype][0], Gen(Dk)
    q, k, v = g.normal(B, L, H, Dk, dtype=T), g.normal(B, L, H, Dk, dtype=T), g.normal(B, L, H, Dv, dtype=T)
    a, beta = -g.uniform(B, L, H, lo=0.0, hi=0.05), g.uniform(B, L, H, lo=0.05, hi=0.95)
    plan = mb.merit_plan_delta_rule(TYPES[dtype][1], B, L, H, H, Dk, Dv, scale=1.0)
    y = mb.merit_delta_rule(plan, q, k, v, a, beta, states=True)[0] if states else mb.merit_delta_rule(plan, q, k, v, a, beta)
    want = om.delta_rule(*(host(t) for t in (q, k, v, a, beta)))[0][:, 16:]     # (the first tokens have few terms)
    unit, size = UNITS[str(y.dtype)], float(np.sqrt(np.mean(want ** 2)))
    small = np.abs(want) <= 2.0 ** -19 / unit * size
    assert small.sum() >= 100
    err = float(np.sqrt(np.mean((host(y)[:, 16:] - want)[small] ** 2)))
    assert err <= 1.01 * unit * float(np.sqrt(np.mean(want[small] ** 2))) + DELTA * 2.0 ** -24 * size, (err / size * 2 ** 24)
