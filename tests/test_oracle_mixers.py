"""oracle/mixers.py: gradients against differences, and the closed forms of small cases."""
import numpy as np
import pytest

from oracle import mixers as om


def _differences(f, args, names, grads, rng, step=1e-5, tol=1e-6):
    """Central differences of f(args) along a few directions against the gradients' dot products."""
    for name in names:
        base = args[name]
        for _ in range(3):
            d = rng.standard_normal(base.shape)
            hi, lo = f({**args, name: base + step * d}), f({**args, name: base - step * d})
            want, got = (hi - lo) / (2 * step), (grads["d" + name] * d).sum()
            assert abs(got - want) <= tol * max(1.0, abs(want)), (name, got, want)


@pytest.mark.parametrize("unit", [True, False])
@pytest.mark.parametrize("lens", [None, [5, 2]])
def test_delta_rule_gradients(unit, lens):
    rng = np.random.default_rng(3)
    B, L, H, K, Dk, Dv = 2, 5, 4, 2, 6, 3
    a = dict(q=rng.standard_normal((B, L, K, Dk)), k=rng.standard_normal((B, L, K, Dk)) * (1 if unit else 0.4),
             v=rng.standard_normal((B, L, H, Dv)), g=-rng.uniform(0.01, 1, (B, L, H)), beta=rng.uniform(0, 1, (B, L, H)),
             h0=rng.standard_normal((B, H, Dk, Dv)))
    dy, dh = rng.standard_normal((B, L, H, Dv)), rng.standard_normal((B, H, Dk, Dv))

    def f(a):
        y, h, _ = om.delta_rule(**a, lens=lens, scale=0.7, unit=unit)
        return (y * dy).sum() + (h * dh).sum()

    grads = om.delta_rule_backward(dy, **a, lens=lens, dh_last=dh, scale=0.7, unit=unit)
    _differences(f, a, ("q", "k", "v", "g", "beta", "h0"), grads, rng)


def test_delta_rule_closed_forms():
    rng = np.random.default_rng(4)
    k, v = rng.standard_normal((1, 3, 1, 4)), rng.standard_normal((1, 3, 1, 2))
    one = np.ones((1, 3, 1))
    # strength 1: a state read along the key that was just written gives its value, whatever came before (unit keys)
    y, _, states = om.delta_rule(k, k, v, -one, one)
    kh = k / np.sqrt((k ** 2).sum(-1, keepdims=True) + om.EPS)
    assert np.allclose(y, v, atol=1e-5)
    # strength 0: only decay
    _, h, _ = om.delta_rule(k, k, v, -one, 0 * one, h0=np.ones((1, 1, 4, 2)))
    assert np.allclose(h, np.exp(-3.0))
    # orthogonal keys, no decay: the sum of outer products
    e = np.eye(4)[None, :3, None]
    _, h, _ = om.delta_rule(e, e, v, None, one, unit=False)
    assert np.allclose(h[0, 0], np.einsum("tk,tv->kv", e[0, :, 0], v[0, :, 0]))
    assert states.shape == (1, 4, 1, 4, 2) and kh.shape == k.shape


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("act", ["none", "silu", "sigmoid"])
@pytest.mark.parametrize("after, before", [(True, True), (True, False), (False, True)])
def test_block_norm_gradients(layer, act, after, before):
    rng = np.random.default_rng(5)
    B, L, C = 2, 3, 7
    a = dict(x=rng.standard_normal((B, L, C)), z=rng.standard_normal((B, L, C)), r=rng.standard_normal((B, L, C)),
             scale=rng.standard_normal(C))
    if after:
        a.update(aw=rng.standard_normal(C), ab=rng.standard_normal(C))
    if before:
        a.update(bw=rng.standard_normal(C), bb=rng.standard_normal(C))
    dout, dn = rng.standard_normal((B, L, C)), rng.standard_normal((B, L, C)) if before else None
    kw = dict(layer=layer, act=act, after=after, before=before)

    def f(a):
        out, n = om.block_norm(**a, **kw)
        return (out * dout).sum() + (0.0 if n is None else (n * dn).sum())

    g = om.block_norm_backward(dout, dn, **a, **kw)
    g.update(daw=g["dafter_weight"], dab=g["dafter_bias"], dbw=g["dbefore_weight"], dbb=g["dbefore_bias"])
    _differences(f, a, tuple(a), g, rng)


def test_block_norm_without_gate_and_stream():
    x = np.random.default_rng(6).standard_normal((1, 2, 50))
    out, n = om.block_norm(x, before=False, eps=0.0)
    assert n is None and np.allclose((out ** 2).mean(-1), 1.0)
    out, n = om.block_norm(x, r=-x, after=False, eps=1e-6)
    assert np.allclose(out, 0.0) and np.allclose(n, 0.0)
