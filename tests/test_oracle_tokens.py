"""The 64-bit definitions of the operators along a sequence of tokens: known values, and every gradient against central
differences (step h = 1e-5: truncation h^2 f''' / 6 and cancellation 1e-16 / h both below 1e-9 of values around one, so 1e-6)."""
import numpy as np
import pytest

from oracle import tokens as ot

H, TOL = 1e-5, 1e-6


def _differences(f, x, weight):
    """The gradient of sum(weight * f(x)) by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += H
        down[i] -= H
        g[i] = ((f(up) - f(down)) * weight).sum() / (2 * H)
    return g


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
def test_group_norm_gradients(kind):
    rng = np.random.default_rng(1)
    x, w, b, dy = rng.normal(size=(2, 3, 6)), rng.normal(size=6), rng.normal(size=6), rng.normal(size=(2, 3, 6))
    dx, dw, db = ot.group_norm_backward(dy, x, 2, w, b, 1e-3, kind)
    for got, value, f in ((dx, x, lambda v: ot.group_norm(v, 2, w, b, 1e-3, kind)[0]),
                          (dw, w, lambda v: ot.group_norm(x, 2, v, b, 1e-3, kind)[0]),
                          (db, b, lambda v: ot.group_norm(x, 2, w, v, 1e-3, kind)[0])):
        np.testing.assert_allclose(got, _differences(f, value, dy), atol=TOL, rtol=TOL)


def test_group_norm_of_a_group_has_mean_0_and_variance_1():
    x = np.random.default_rng(2).normal(5.0, 3.0, size=(2, 50, 8))
    y, mean, rstd = ot.group_norm(x, 4, eps=0.0)
    v = y.reshape(2, 50, 4, 2)
    np.testing.assert_allclose(v.mean(axis=(1, 3)), 0.0, atol=1e-12)
    np.testing.assert_allclose((v ** 2).mean(axis=(1, 3)), 1.0, rtol=1e-12)
    np.testing.assert_allclose(mean[0, 1], x[0, :, 2:4].mean(), rtol=1e-12)


@pytest.mark.parametrize("kind", ["none", "silu"])
def test_causal_conv_gradients(kind):
    rng = np.random.default_rng(3)
    B, L, D, K = 2, 5, 2, 3
    x, w, b = rng.normal(size=(B, L, D)), rng.normal(size=(D, K)), rng.normal(size=D)
    init, dy, dfinal = rng.normal(size=(B, K - 1, D)), rng.normal(size=(B, L, D)), rng.normal(size=(B, K - 1, D))
    lens = [5, 1]

    def both(x_, w_, b_, i_):
        y, f = ot.causal_conv(x_, w_, b_, i_, lens, kind)
        return np.concatenate([y.ravel(), f.ravel()])

    weight = np.concatenate([dy.ravel(), dfinal.ravel()])
    got = ot.causal_conv_backward(dy, x, w, b, init, lens, dfinal, kind)
    for g, value, f in zip(got, (x, w, b, init), (lambda v: both(v, w, b, init), lambda v: both(x, v, b, init),
                                                  lambda v: both(x, w, v, init), lambda v: both(x, w, b, v))):
        np.testing.assert_allclose(g, _differences(f, value, weight), atol=TOL, rtol=TOL)


def test_causal_conv_is_causal_and_continues():
    rng = np.random.default_rng(4)
    x, w = rng.normal(size=(1, 9, 3)), rng.normal(size=(3, 4))
    y, final = ot.causal_conv(x, w)
    y1, f1 = ot.causal_conv(x[:, :2], w)
    y2, f2 = ot.causal_conv(x[:, 2:], w, init=f1)
    np.testing.assert_allclose(np.concatenate([y1, y2], 1), y, rtol=1e-14)
    np.testing.assert_array_equal(f2, final)
    np.testing.assert_allclose(y[0, 0], w[:, 3] * x[0, 0])


@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("gate", [True, False])
def test_scan_gradients(softplus, gate):
    rng = np.random.default_rng(5)
    B, L, D, N, G = 2, 4, 4, 2, 2
    v = dict(x=rng.normal(size=(B, L, D)), dt=rng.uniform(0.1, 1.0, size=(B, L, D)), A=-rng.uniform(0.2, 2.0, size=(D, N)),
             Bm=rng.normal(size=(B, L, G, N)), Cm=rng.normal(size=(B, L, G, N)), skip=rng.normal(size=D),
             z=rng.normal(size=(B, L, D)) if gate else None, dt_bias=rng.normal(0, 0.1, size=D), h0=rng.normal(size=(B, D, N)))
    lens, dy, dh = [4, 2], rng.normal(size=(B, L, D)), rng.normal(size=(B, D, N))

    def both(**new):
        y, h, _ = ot.scan(**{**v, **new}, lens=lens, softplus=softplus)
        return np.concatenate([y.ravel(), h.ravel()])

    weight = np.concatenate([dy.ravel(), dh.ravel()])
    got = ot.scan_backward(dy, **v, lens=lens, dh_last=dh, softplus=softplus)
    names = dict(x="dx", dt="ddt", A="dA", Bm="dB", Cm="dC", skip="dskip", z="dz", dt_bias="ddt_bias", h0="dh0")
    for k, name in names.items():
        if v[k] is not None:
            np.testing.assert_allclose(got[name], _differences(lambda a: both(**{k: a}), v[k], weight), atol=TOL, rtol=TOL)


def test_scan_of_constant_input_reaches_its_limit():
    """h = a h + s x B settles at s x B / (1 - a)."""
    L, s, A = 400, 0.1, -1.5
    y, h, _ = ot.scan(np.full((1, L, 1), 2.0), np.full((1, L, 1), s), np.full((1, 1), A), np.full((1, L, 1, 1), 3.0),
                      np.full((1, L, 1, 1), 0.5), softplus=False)
    limit = s * 2.0 * 3.0 / (1 - np.exp(s * A))
    assert abs(h[0, 0, 0] - limit) < 1e-12 and abs(y[0, -1, 0] - 0.5 * limit) < 1e-12
