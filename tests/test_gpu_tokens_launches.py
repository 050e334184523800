"""Token operators over more workgroups than one launch holds (fewer than 2^32 threads), against the definition in 64 bits
(tolerances: token_helpers)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from token_helpers import DEV, TYPES, Gen, check, host     # noqa: E402


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("B, G", [(1 << 20, 8), (8200, 1024)])
def test_scan_over_many_short_sequences(mb, B, G):
    """Two tokens, one state, a channel a group.  Chain: 4 L + N + 16."""
    L, N = 2, 1
    T, code, _ = TYPES["bf16"]
    g = Gen(21)
    x, dt, z, Bm, Cm = (g.normal(B, L, G, dtype=T) for _ in range(5))
    A, skip, h0 = -g.uniform(G, N, lo=0.1, hi=4.0), g.normal(G), g.normal(B, G, N)
    lens = torch.from_numpy(g.rng.integers(0, L + 1, size=B).astype(np.int32)).to(DEV)
    plan = mb.merit_plan_scan(code, B, L, G, N, G)
    assert plan.kernel() == "merit_scan_tiles+merit_scan_tiles"
    y, h = mb.merit_scan(plan, x, dt, A, Bm[..., None], Cm[..., None], skip=skip, z=z, h0=h0, lens=lens, final=True)
    x, dt, z, Bm, Cm, A, skip, state = (host(t) for t in (x, dt, z, Bm, Cm, A[:, 0], skip, h0[..., 0]))
    n, want = lens.cpu().numpy()[:, None], np.zeros((B, L, G))
    for t in range(L):
        s = np.logaddexp(0.0, dt[:, t])
        state = np.where(t < n, np.exp(s * A) * state + s * x[:, t] * Bm[:, t], state)
        want[:, t] = np.where(t < n, (Cm[:, t] * state + skip * x[:, t]) * z[:, t] / (1.0 + np.exp(-z[:, t])), 0.0)
    check(y, want, 4 * L + N + 16, "y")
    check(h, state[..., None], 4 * L + N + 16, "h")
