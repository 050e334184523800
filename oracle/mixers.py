"""The gated delta rule and the norms before and after a block in 64 bits, from their definitions: numpy, token by token.
Shares no code with the kernels; gradients are the formulas' own and are pinned against differences (test_oracle_mixers)."""
import numpy as np

from .tokens import _f64

EPS = 1e-6


def _direction(x, unit):
    """(x over its length, one over the length)"""
    r = 1.0 / np.sqrt((x * x).sum(-1, keepdims=True) + EPS) if unit else np.ones(x.shape[:-1] + (1,))
    return x * r, r


def _tokens(lens, b, L):
    return L if lens is None else min(max(int(lens[b]), 0), L)


# ---- gated delta rule: q, k[B, L, K, Dk], v[B, L, H, Dv], g, beta[B, L, H] ------------------------------------
def delta_rule(q, k, v, g, beta, h0=None, lens=None, scale=1.0, unit=True):
    """(y, the state behind the last token, all states [B, L + 1, H, Dk, Dv])"""
    q, k, v, g, beta, h0 = _f64(q, k, v, g, beta, h0)
    (B, L, H, Dv), K, Dk = v.shape, k.shape[2], k.shape[3]
    head = np.arange(H) // (H // K)
    (q, _), (k, _) = _direction(q, unit), _direction(k, unit)
    y, last, states = np.zeros(v.shape), np.zeros((B, H, Dk, Dv)), np.zeros((B, L + 1, H, Dk, Dv))
    for b in range(B):
        S = np.zeros((H, Dk, Dv)) if h0 is None else h0[b].copy()
        states[b, 0] = S
        for t in range(_tokens(lens, b, L)):
            kt, qt = k[b, t, head], q[b, t, head]
            S = S if g is None else S * np.exp(g[b, t])[:, None, None]
            u = beta[b, t][:, None] * (v[b, t] - (S * kt[:, :, None]).sum(1))
            S = S + kt[:, :, None] * u[:, None, :]
            states[b, t + 1] = S
            y[b, t] = scale * (S * qt[:, :, None]).sum(1)
        last[b] = S
    return y, last, states


def delta_rule_backward(dy, q, k, v, g, beta, h0=None, lens=None, dh_last=None, scale=1.0, unit=True):
    """{'dq', 'dk', 'dv', 'dg', 'dbeta', 'dh0'}"""
    _, _, states = delta_rule(q, k, v, g, beta, h0, lens, scale, unit)
    dy, q, k, v, g, beta, dh_last = _f64(dy, q, k, v, g, beta, dh_last)
    (B, L, H, Dv), K, Dk = v.shape, k.shape[2], k.shape[3]
    head = np.arange(H) // (H // K)
    (qh, rq), (kh, rk) = _direction(q, unit), _direction(k, unit)
    dq, dk, dv, dg, db = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(beta.shape), np.zeros(beta.shape)
    dh0 = np.zeros((B, H, Dk, Dv))
    for b in range(B):
        D = np.zeros((H, Dk, Dv)) if dh_last is None else dh_last[b].copy()
        for t in reversed(range(_tokens(lens, b, L))):
            kt, qt, S = kh[b, t, head], qh[b, t, head], states[b, t + 1]
            np.add.at(dq[b, t], head, scale * (S * dy[b, t][:, None, :]).sum(2))
            D = D + scale * qt[:, :, None] * dy[b, t][:, None, :]
            a = np.ones(H) if g is None else np.exp(g[b, t])
            faded = states[b, t] * a[:, None, None]
            miss = v[b, t] - (faded * kt[:, :, None]).sum(1)
            du = (D * kt[:, :, None]).sum(1)
            db[b, t] = (du * miss).sum(1)
            dmiss = du * beta[b, t][:, None]
            dv[b, t] = dmiss
            np.add.at(dk[b, t], head, (D * (beta[b, t][:, None] * miss)[:, None, :]).sum(2) - (faded * dmiss[:, None, :]).sum(2))
            D = D - kt[:, :, None] * dmiss[:, None, :]
            dg[b, t] = (D * faded).sum((1, 2))
            D = D * a[:, None, None]
        dh0[b] = D
    if unit:
        dq = rq * (dq - qh * (qh * dq).sum(-1, keepdims=True))
        dk = rk * (dk - kh * (kh * dk).sum(-1, keepdims=True))
    return {"dq": dq, "dk": dk, "dv": dv, "dg": dg, "dbeta": db, "dh0": dh0}


# ---- the norms before and after a block: x[B, L, C] ------------------------------------------------------------
def _gate(z, act):
    p = 1.0 / (1.0 + np.exp(-z))
    return {"none": z, "relu": np.maximum(z, 0.0), "silu": z * p, "sigmoid": p}[act]


def _gate_slope(z, act):
    p = 1.0 / (1.0 + np.exp(-z))
    return {"none": np.ones_like(z), "relu": (z > 0) * 1.0, "silu": p + z * p * (1.0 - p), "sigmoid": p * (1.0 - p)}[act]


def _norm(x, layer, eps):
    """(norm(x), one over the root, the mean)"""
    m = x.mean(-1, keepdims=True) if layer else np.zeros(x.shape[:-1] + (1,))
    r = 1.0 / np.sqrt(((x - m) ** 2).mean(-1, keepdims=True) + eps)
    return (x - m) * r, r, m


def _norm_back(d, xh, r, layer):
    return r * (d - (d.mean(-1, keepdims=True) if layer else 0.0) - xh * (d * xh).mean(-1, keepdims=True))


def block_norm(x, z=None, r=None, aw=None, ab=None, scale=None, bw=None, bb=None, layer=False, eps=1e-6, act="none", after=True,
               before=True):
    """(out, n or None)"""
    x, z, r, aw, ab, scale, bw, bb = _f64(x, z, r, aw, ab, scale, bw, bb)
    u = _norm(x, layer, eps)[0] if after else x
    u = u * (1.0 if aw is None else aw) + (0.0 if ab is None else ab)
    t = u if z is None else u * _gate(z, act)
    out = (0.0 if r is None else r) + (1.0 if scale is None else scale) * t
    if not before:
        return out, None
    return out, _norm(out, layer, eps)[0] * (1.0 if bw is None else bw) + (0.0 if bb is None else bb)


def block_norm_backward(dout, dn, x, z=None, r=None, aw=None, ab=None, scale=None, bw=None, bb=None, layer=False, eps=1e-6,
                        act="none", after=True, before=True):
    """{'dx', 'dz', 'dr', 'dafter_weight', 'dafter_bias', 'dscale', 'dbefore_weight', 'dbefore_bias'}"""
    dout, dn, x, z, r, aw, ab, scale, bw = _f64(dout, dn, x, z, r, aw, ab, scale, bw)
    xh, rx, _ = _norm(x, layer, eps) if after else (x, None, None)
    u = xh * (1.0 if aw is None else aw) + (0.0 if ab is None else ab)
    e = np.ones_like(x) if z is None else _gate(z, act)
    s = 1.0 if scale is None else scale
    out = (0.0 if r is None else r) + s * u * e
    do = np.zeros_like(x) if dout is None else dout.copy()
    res = {"dbefore_weight": np.zeros(x.shape[2]), "dbefore_bias": np.zeros(x.shape[2])}
    if before:
        oh, ro, _ = _norm(out, layer, eps)
        do += _norm_back(dn * (1.0 if bw is None else bw), oh, ro, layer)
        res["dbefore_weight"], res["dbefore_bias"] = (dn * oh).sum((0, 1)), dn.sum((0, 1))
    du = do * s * e
    res.update(dr=do, dscale=(do * u * e).sum((0, 1)), dz=None if z is None else do * s * u * _gate_slope(z, act),
               dafter_weight=(du * xh).sum((0, 1)), dafter_bias=du.sum((0, 1)))
    res["dx"] = _norm_back(du * (1.0 if aw is None else aw), xh, rx, layer) if after else du
    return res
