"""How many digits the delta rule's fp32 arithmetic keeps, where a result shows them: sums that cancel, decays by themselves,
products of values with all of their bits set."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from mixer_helpers import DELTA, UNITS          # noqa: E402
from oracle import mixers as om                 # noqa: E402
from token_helpers import DEV, TYPES, Gen, host     # noqa: E402


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


def test_decays_by_themselves(mb):
    """exp(g) to fp32: the exponential function's one step of 2^-23, a rounding of its argument below one, and one of the product.
    What goes through a product of bfloat16 terms has besides what the third one loses, which lies at 2^-16 of the value: bfloat16 has
    steps of 2^-133 below 2^-126, so of values below 2^-110 the term loses half such a step where it is rounded (P, in y), up to a
    whole one where it is cut off (what a state takes up)."""
    H = 512
    g = -torch.linspace(0.001, 80.0, H, dtype=torch.float64).float().to(DEV)
    want = np.exp(host(g))

    def near(got, what, term=0.0):
        err = np.abs(host(got).reshape(H, -1) - want[:, None]) / (4.0 * 2.0 ** -24 * want[:, None] + term)
        assert err.max() <= 1.0, (what, float(err.max()))

    zero, one = torch.zeros(1, H, 1, device=DEV), torch.ones(1, H, 1, device=DEV)
    # a token more: nothing is written, the state fades
    step = mb.merit_plan_delta_rule(mb.MERIT_F32, 1, 1, H, H, 1, 1, scale=1.0, normalize=False)
    y, h = mb.merit_delta_rule_step(step, one[..., None], one, one, zero, g[None], zero[..., 0])
    near(h, "a token's state")
    near(y, "a token's result")
    # two tokens of a prompt: the second reads what the first wrote, and what was there before; both fade on the way
    plan = mb.merit_plan_delta_rule(mb.MERIT_F32, 1, 2, H, H, 2, 1, scale=1.0, normalize=False)
    k = torch.zeros(1, 2, H, 2, device=DEV)
    k[:, 0, :, 0] = 1.0
    v, beta = torch.ones(1, 2, H, 1, device=DEV), torch.zeros(1, 2, H, device=DEV)
    beta[:, 0] = 1.0
    gates = torch.stack([torch.zeros_like(g), g])[None]
    h0 = torch.zeros(1, H, 2, 1, device=DEV)
    h0[:, :, 1] = 1.0
    for axis, what, term in ((0, "written", 2.0 ** -134), (1, "from before", 0.0)):
        q = torch.zeros(1, 2, H, 2, device=DEV)
        q[..., axis] = 1.0
        y, h = mb.merit_delta_rule(plan, q, k, v, gates, beta, h0=h0, final=True)
        near(y[0, 1], what, term)
        near(h[0, :, axis], what + ", state", 2.0 * term)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_products_of_values_with_all_bits_set(mb, dtype):
    """1 + a / 128 - 2^-23: cut after eight bits, and after eight more, such a value leaves as much as it can.  A product of two is
    a handful of fp32 sums of one sign, so nothing but the last one's rounding, or its cut, is of any size: two of 2^-24; a binary16
    factor (1 + a / 128 - 2^-10) is in two terms and leaves nothing."""
    H = 64
    T, last = (torch.float32, 2.0 ** -23) if dtype == "f32" else (torch.float16, 2.0 ** -10)
    a = torch.arange(1, 9, dtype=torch.float64) / 128
    s, q = (1 + a - 2.0 ** -23).repeat_interleave(8), (1 + a - last).repeat(8)
    h0, qd = s.float().view(1, H, 1, 1).to(DEV), q.to(T).view(1, 1, H, 1).to(DEV)
    plan = mb.merit_plan_delta_rule(TYPES[dtype][1], 1, 1, H, H, 1, 1, scale=1.0, normalize=False)
    none, v = torch.zeros(1, 1, H, device=DEV), torch.zeros(1, 1, H, 1, dtype=T, device=DEV)
    # read by q: y of fp32 shows it, and what a key of the same value takes away from v, which the state keeps
    if dtype == "f32":
        y = mb.merit_delta_rule(plan, qd, torch.zeros_like(qd), v, None, none, h0=h0)
        err = np.abs(host(y).ravel() / (s * q).numpy() - 1.0).max() * 2 ** 24
        assert err <= 4.0, float(err)
    one = torch.ones_like(none)
    h = mb.merit_delta_rule(plan, torch.zeros_like(qd), qd, v, None, one, h0=h0, final=True)[1]
    # S - q (q S): the products' cuts and roundings, of q S and of q (q S), and the difference's
    inner = (s * q).numpy()
    err = np.abs(host(h).ravel() - (s.numpy() - q.numpy() * inner)) / (q.numpy() * inner) * 2 ** 24
    assert err.max() <= 6.0, float(err.max())
