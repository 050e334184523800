"""Infinities in what a group's channels share, where the channels do not fill their workgroup: what the definition says about
them, and nothing from lanes that have no channel."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import tokens as ot                        # noqa: E402
from token_helpers import DEV, TYPES, Gen, check, host     # noqa: E402


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("D, G", [(10, 1), (64, 1), (70, 1), (6, 2)])
@pytest.mark.parametrize("N", [1, 3, 8, 16, 17, 64])
@pytest.mark.parametrize("what", ["B", "C"])
def test_gradients_of_tokens(mb, what, N, D, G):
    """All operands positive, so that no sum of the definition has infinities of both signs: a result is infinite, or it is as
    near as ever, and a NaN only where the definition has one (0 times an infinite state).  Chain: 3 (4 L + N + 16) + D / G."""
    B, L = 2, 37
    g = Gen(31)
    u = {k: g.uniform(*s, lo=0.2, hi=1.0) for k, s in dict(x=(B, L, D), dt=(B, L, D), B=(B, L, G, N), C=(B, L, G, N), dy=(B, L, D)).items()}
    A = -g.uniform(D, N, lo=0.1, hi=2.0)
    u[what][1, 20, G - 1, N - 1] = float("inf")
    plan = mb.merit_plan_scan(TYPES["f32"][1], B, L, D, N, G)
    _, st = mb.merit_scan(plan, u["x"], u["dt"], A, u["B"], u["C"], states=True)
    got = mb.merit_scan_backward(plan, u["dy"], u["x"], u["dt"], A, u["B"], u["C"], st)
    with np.errstate(invalid="ignore"):
        want = ot.scan_backward(host(u["dy"]), host(u["x"]), host(u["dt"]), host(A), host(u["B"]), host(u["C"]))
    for k in ("dx", "ddt", "dB", "dC"):
        w, t = want[k], host(got[k])
        assert np.array_equal(np.isnan(t), np.isnan(w)), k
        far = np.isinf(w)
        assert np.array_equal(t[far], w[far]), k
        finite = np.isfinite(w)
        check(got[k].cpu()[torch.from_numpy(finite)], w[finite], 3 * (4 * L + N + 16) + D // G, k)
    assert np.isinf(want["dC" if what == "B" else "dB"]).any()


@pytest.mark.parametrize("L, lens", [(37, None), (48, None), (48, (48, 40, 17))])
@pytest.mark.parametrize("N", [1, 3, 16, 64])
@pytest.mark.parametrize("last", [True, False])
def test_gradient_of_decays(mb, last, N, L, lens):
    """A state that becomes infinite at a sequence's last token has no part in dA (the decays multiply the states before it);
    one that does so earlier makes that entry infinite.  Chain: 3 (4 L + N + 16) + B L."""
    B, D = 3, 20
    g = Gen(32)
    u = {k: g.uniform(*s, lo=0.2, hi=1.0) for k, s in dict(x=(B, L, D), dt=(B, L, D), B=(B, L, 1, N), C=(B, L, 1, N), dy=(B, L, D)).items()}
    A = -g.uniform(D, N, lo=0.1, hi=2.0)
    ends = [L] * B if lens is None else lens
    u["x"][1, ends[1] - 1 if last else 9, 5] = float("inf")
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    plan = mb.merit_plan_scan(TYPES["f32"][1], B, L, D, N)
    _, st = mb.merit_scan(plan, u["x"], u["dt"], A, u["B"], u["C"], lens=n, states=True)
    got = host(mb.merit_scan_backward(plan, u["dy"], u["x"], u["dt"], A, u["B"], u["C"], st, lens=n)["dA"])
    with np.errstate(invalid="ignore"):
        want = ot.scan_backward(*(host(u[k]) for k in ("dy", "x", "dt")), host(A), host(u["B"]), host(u["C"]), lens=ends)["dA"]
    assert np.isfinite(want).all() if last else np.isinf(want[5]).all() and np.isfinite(np.delete(want, 5, 0)).all()
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    finite = np.isfinite(want)
    check(torch.from_numpy(got[finite]).float(), want[finite], 3 * (4 * L + N + 16) + B * L, "dA")


@pytest.mark.parametrize("N", [1, 3, 16, 64])
def test_an_infinite_state_through_chunks(mb, N):
    """An infinite state stays one, however much of it has decayed: also where a sequence runs in chunks, over which the decay is
    less than fp32 can hold (steps of at least 0.31 and A of -12: 5 to 11 bits a token)."""
    B, L, D = 1, 400, 20
    g = Gen(33)
    u = {k: g.uniform(*s, lo=0.2, hi=1.0) for k, s in dict(x=(B, L, D), dt=(B, L, D), B=(B, L, 1, N), C=(B, L, 1, N), dy=(B, L, D)).items()}
    u["dt"] -= 1.2
    A = torch.full((D, N), -12.0, device=DEV)
    plan = mb.merit_plan_scan(TYPES["f32"][1], B, L, D, N)
    assert "+" in plan.kernel() and plan.kernel(mb.MERIT_PASS_BACKWARD).startswith("merit_scan_back_chunks")
    x, dy = u["x"].clone(), u["dy"].clone()
    x[0, 7, 4] = dy[0, 390, 9] = float("inf")
    y, h = mb.merit_scan(plan, x, u["dt"], A, u["B"], u["C"], final=True)
    clean, _ = mb.merit_scan(plan, u["x"], u["dt"], A, u["B"], u["C"], final=True)
    assert torch.isposinf(y[0, 7:, 4]).all() and torch.isposinf(h[0, 4]).all()
    y[0, 7:, 4] = clean[0, 7:, 4]
    assert torch.equal(y, clean)
    _, st = mb.merit_scan(plan, u["x"], u["dt"], A, u["B"], u["C"], states=True)
    got = mb.merit_scan_backward(plan, dy, u["x"], u["dt"], A, u["B"], u["C"], st, dh0=True)
    clean = mb.merit_scan_backward(plan, u["dy"], u["x"], u["dt"], A, u["B"], u["C"], st, dh0=True)
    assert torch.isposinf(got["dx"][0, :391, 9]).all() and torch.isposinf(got["dh0"][0, 9]).all()
    got["dx"][0, :391, 9] = clean["dx"][0, :391, 9]
    assert torch.equal(got["dx"], clean["dx"])
