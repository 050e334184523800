"""The operators along a sequence of tokens in 64 bits, from their definitions: numpy, token by token and group by group.
Shares no code with the kernels; gradients are the formulas' own and are pinned against differences (test_oracle_tokens)."""
import numpy as np


def act(u, kind):
    if kind == "silu":
        return u / (1.0 + np.exp(-u))
    return np.maximum(u, 0.0) if kind == "relu" else u


def act_slope(u, kind):
    if kind == "silu":
        p = 1.0 / (1.0 + np.exp(-u))
        return p * (1.0 + u * (1.0 - p))
    return (u > 0).astype(np.float64) if kind == "relu" else np.ones_like(u)


def _f64(*arrays):
    return [None if a is None else np.asarray(a, dtype=np.float64) for a in arrays]


# ---- group norm: x[N, S, C] ---------------------------------------------------------------------
def group_norm(x, groups, weight=None, bias=None, eps=1e-5, kind="none"):
    """(y, mean[N, groups], rstd[N, groups])"""
    x, weight, bias = _f64(x, weight, bias)
    N, S, C = x.shape
    v = x.reshape(N, S, groups, C // groups)
    mean = v.mean(axis=(1, 3))
    rstd = 1.0 / np.sqrt(((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3)) + eps)
    u = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(N, S, C)
    u = u * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)
    return act(u, kind), mean, rstd


def group_norm_backward(dy, x, groups, weight=None, bias=None, eps=1e-5, kind="none"):
    """(dx, dweight, dbias)"""
    dy, x, weight, bias = _f64(dy, x, weight, bias)
    N, S, C = x.shape
    _, mean, rstd = group_norm(x, groups, eps=eps)
    xh = ((x.reshape(N, S, groups, -1) - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(N, S, C)
    w = np.ones(C) if weight is None else weight
    du = dy * act_slope(xh * w + (0.0 if bias is None else bias), kind)
    g, h = (du * w).reshape(N, S, groups, -1), xh.reshape(N, S, groups, -1)
    m1, m2 = g.mean(axis=(1, 3), keepdims=True), (g * h).mean(axis=(1, 3), keepdims=True)
    dx = (rstd[:, None, :, None] * (g - m1 - h * m2)).reshape(N, S, C)
    return dx, (du * xh).sum(axis=(0, 1)), du.sum(axis=(0, 1))


# ---- short causal convolution: x[B, L, D], weight[D, K] -----------------------------------------------
def _tokens(x, init, K, b, n):
    """(init, x) of sequence b up to its n tokens: [K - 1 + n, D]"""
    first = np.zeros((K - 1, x.shape[2])) if init is None else init[b]
    return np.concatenate([first, x[b, :n]], axis=0)


def causal_conv(x, weight, bias=None, init=None, lens=None, kind="none"):
    """(y, the last K - 1 tokens)"""
    x, weight, bias, init = _f64(x, weight, bias, init)
    (B, L, D), K = x.shape, weight.shape[1]
    y, final = np.zeros((B, L, D)), np.zeros((B, K - 1, D))
    for b in range(B):
        n = L if lens is None else min(max(int(lens[b]), 0), L)
        rows = _tokens(x, init, K, b, n)
        for t in range(n):
            u = np.zeros(D) if bias is None else bias.copy()
            for a in range(K):
                u = u + weight[:, a] * rows[t + a]
            y[b, t] = act(u, kind)
        final[b] = rows[n:n + K - 1]
    return y, final


def causal_conv_backward(dy, x, weight, bias=None, init=None, lens=None, dfinal=None, kind="none"):
    """(dx, dweight, dbias, dinit)"""
    dy, x, weight, bias, init, dfinal = _f64(dy, x, weight, bias, init, dfinal)
    (B, L, D), K = x.shape, weight.shape[1]
    dx, dw, db, dinit = np.zeros((B, L, D)), np.zeros((D, K)), np.zeros(D), np.zeros((B, K - 1, D))
    for b in range(B):
        n = L if lens is None else min(max(int(lens[b]), 0), L)
        rows = _tokens(x, init, K, b, n)
        drows = np.zeros_like(rows)
        for t in range(n):
            u = np.zeros(D) if bias is None else bias.copy()
            for a in range(K):
                u = u + weight[:, a] * rows[t + a]
            du = dy[b, t] * act_slope(u, kind)
            db += du
            for a in range(K):
                dw[:, a] += du * rows[t + a]
                drows[t + a] += du * weight[:, a]
        if dfinal is not None:
            drows[n:n + K - 1] += dfinal[b]
        dinit[b], dx[b, :n] = drows[:K - 1], drows[K - 1:]
    return dx, dw, db, dinit


# ---- selective scan: x[B, L, D], A[D, N], B and C [B, L, G, N] --------------------------------------------
def _steps(dt, dt_bias, softplus):
    v = dt if dt_bias is None else dt + dt_bias
    return v, (np.logaddexp(0.0, v) if softplus else v)


def scan(x, dt, A, Bm, Cm, skip=None, z=None, dt_bias=None, h0=None, lens=None, softplus=True):
    """(y, the state behind the last token, all states [B, L, D, N])"""
    x, dt, A, Bm, Cm, skip, z, dt_bias, h0 = _f64(x, dt, A, Bm, Cm, skip, z, dt_bias, h0)
    (B, L, D), N, G = x.shape, A.shape[1], Bm.shape[2]
    group = np.arange(D) // (D // G)
    _, step = _steps(dt, dt_bias, softplus)
    y, last, states = np.zeros((B, L, D)), np.zeros((B, D, N)), np.zeros((B, L, D, N))
    for b in range(B):
        h = np.zeros((D, N)) if h0 is None else h0[b].copy()
        for t in range(L if lens is None else min(max(int(lens[b]), 0), L)):
            s = step[b, t][:, None]
            h = np.exp(s * A) * h + s * x[b, t][:, None] * Bm[b, t, group]
            states[b, t] = h
            y[b, t] = (h * Cm[b, t, group]).sum(-1) + (0.0 if skip is None else skip * x[b, t])
            if z is not None:
                y[b, t] *= act(z[b, t], "silu")
        last[b] = h
    return y, last, states


def scan_backward(dy, x, dt, A, Bm, Cm, skip=None, z=None, dt_bias=None, h0=None, lens=None, dh_last=None, softplus=True):
    """{'dx', 'ddt', 'dB', 'dC', 'dz', 'dA', 'dskip', 'ddt_bias', 'dh0'}"""
    _, _, states = scan(x, dt, A, Bm, Cm, skip, z, dt_bias, h0, lens, softplus)
    dy, x, dt, A, Bm, Cm, skip, z, dt_bias, h0, dh_last = _f64(dy, x, dt, A, Bm, Cm, skip, z, dt_bias, h0, dh_last)
    (B, L, D), N, G = x.shape, A.shape[1], Bm.shape[2]
    group = np.arange(D) // (D // G)
    v, step = _steps(dt, dt_bias, softplus)
    dx, ddt, dz = np.zeros((B, L, D)), np.zeros((B, L, D)), np.zeros((B, L, D))
    dB, dC, dA = np.zeros(Bm.shape), np.zeros(Cm.shape), np.zeros((D, N))
    dskip, dbias, dh0 = np.zeros(D), np.zeros(D), np.zeros((B, D, N))
    for b in range(B):
        carry = np.zeros((D, N)) if dh_last is None else dh_last[b].copy()
        for t in reversed(range(L if lens is None else min(max(int(lens[b]), 0), L))):
            g = dy[b, t]
            if z is not None:
                y0 = (states[b, t] * Cm[b, t, group]).sum(-1) + (0.0 if skip is None else skip * x[b, t])
                dz[b, t] = g * y0 * act_slope(z[b, t], "silu")
                g = g * act(z[b, t], "silu")
            s = step[b, t][:, None]
            a = np.exp(s * A)
            before = states[b, t - 1] if t else (np.zeros((D, N)) if h0 is None else h0[b])
            lam = carry + g[:, None] * Cm[b, t, group]
            q = lam * a * before
            into = (lam * Bm[b, t, group]).sum(-1)
            dx[b, t] = into * step[b, t] + (0.0 if skip is None else skip * g)
            d = into * x[b, t] + (q * A).sum(-1)
            ddt[b, t] = d / (1.0 + np.exp(-v[b, t])) if softplus else d
            dA += q * s
            np.add.at(dB[b, t], group, lam * s * x[b, t][:, None])
            np.add.at(dC[b, t], group, states[b, t] * g[:, None])
            dskip += g * x[b, t]
            dbias += ddt[b, t]
            carry = lam * a
        dh0[b] = carry
    return {"dx": dx, "ddt": ddt, "dB": dB, "dC": dC, "dz": dz, "dA": dA, "dskip": dskip, "ddt_bias": dbias, "dh0": dh0}
