"""The gated delta rule, and the norms before and after a block with its gate and residual scale (include/merit_tokens.h):
operators along a sequence of tokens like those of `tokens`, called the same way.  `binding` re-exports everything here.
"""
from __future__ import annotations

import ctypes

from .tokens import MERIT_ACT_NONE, TokenPlan, _binding, _bits, _call, _F32, _I32, _P, _T

MERIT_ACT_SIGMOID = 3                   # the gate of merit_block_norm only
MERIT_DELTA_MAX_KEYS = 128
MERIT_DELTA_CHUNK = 64
MERIT_DELTA_KEPT = 9728
MERIT_BLOCK_NORM_MAX_CHANNELS = 8192

_ENTRIES = ("merit_delta_rule", "merit_delta_rule_backward", "merit_delta_rule_step", "merit_block_norm", "merit_block_norm_backward")


def _declare(L):
    """Argument types of the entry points (binding.lib() calls this once)."""
    P, i64, c_int, f64, PP = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_double, ctypes.POINTER(ctypes.c_void_p)
    L.merit_plan_delta_rule.argtypes = [c_int] + [i64] * 6 + [f64, c_int, PP]
    L.merit_plan_block_norm.argtypes = [c_int, c_int] + [i64] * 3 + [f64] + [c_int] * 4 + [PP]
    for name in _ENTRIES:
        getattr(L, name).argtypes = [P, P, P, i64, P]
    for name in _ENTRIES + ("merit_plan_delta_rule", "merit_plan_block_norm"):
        getattr(L, name).restype = c_int


# --------------------------------------------------------------------------
# gated delta rule
# --------------------------------------------------------------------------
def merit_plan_delta_rule(dtype, B, L, heads, key_heads, Dk, Dv, *, scale=None, normalize=True) -> TokenPlan:
    """q, k[B, L, key_heads, Dk], v[B, L, heads, Dv]; scale: of the results, Dk^-1/2 if not given; normalize: q and k count by
    their direction."""
    b, h = _binding(), ctypes.c_void_p()
    scale = max(Dk, 1) ** -0.5 if scale is None else float(scale)
    b._check(b.lib().merit_plan_delta_rule(dtype, B, L, heads, key_heads, Dk, Dv, scale, int(bool(normalize)), ctypes.byref(h)),
             "merit_plan_delta_rule")
    qk, v, gate, state = (B, L, key_heads, Dk), (B, L, heads, Dv), (B, L, heads), (B, heads, Dk, Dv)
    kept = (B, -(-L // MERIT_DELTA_CHUNK), heads, -(-(MERIT_DELTA_KEPT + (Dk + MERIT_DELTA_CHUNK) * Dv) // 4) * 4)
    qk1, v1, gate1 = (B, key_heads, Dk), (B, heads, Dv), (B, heads)
    return TokenPlan(h, dtype, {
        "merit_delta_rule": (0, [("q", _T, qk, 2, "in"), ("k", _T, qk, 2, "in"), ("v", _T, v, 2, "in"), ("g", _F32, gate, 2, "opt"),
                                 ("beta", _P, gate, 2, "in"), ("h0", _F32, state, 0, "opt"), ("lens", _I32, (B,), 0, "opt"),
                                 ("y", _T, v, 2, "out"), ("h_last", _F32, state, 0, "out?"), ("states", _F32, kept, 0, "out?")]),
        "merit_delta_rule_backward": (1, [("dy", _T, v, 2, "in"), ("q", _T, qk, 2, "in"), ("k", _T, qk, 2, "in"),
                                          ("g", _F32, gate, 2, "opt"), ("beta", _P, gate, 2, "in"), ("states", _F32, kept, 0, "in"),
                                          ("lens", _I32, (B,), 0, "opt"), ("dh_last", _F32, state, 0, "opt"),
                                          ("dq", _T, qk, 2, "out"), ("dk", _T, qk, 2, "out"), ("dv", _T, v, 2, "out"),
                                          ("dg", _F32, gate, 2, "out?"), ("dbeta", _F32, gate, 2, "out"),
                                          ("dh0", _F32, state, 0, "out?")]),
        "merit_delta_rule_step": (2, [("h", _F32, state, 0, "in"), ("q", _T, qk1, 1, "in"), ("k", _T, qk1, 1, "in"),
                                      ("v", _T, v1, 1, "in"), ("g", _F32, gate1, 1, "opt"), ("beta", _P, gate1, 1, "in"),
                                      ("y", _T, v1, 1, "out"), ("h_out", _F32, state, 0, "out")])})


def merit_delta_rule(plan, q, k, v, g, beta, *, h0=None, lens=None, final=False, states=False, y=None, stream=None):
    """y[, the state behind the last token][, what the backward pass takes].  g: the logarithm of the decay (None: no decay);
    final: True, or a tensor, which may be h0."""
    given = None if isinstance(final, bool) else final
    on = final is not False
    r = _call(plan, "merit_delta_rule", (q, k, v, g, beta, h0, lens, y, given, None), 0x80 | on << 8 | bool(states) << 9, stream)
    return r[0] if not (on or states) else tuple(t for t, w in zip(r, (True, on, states)) if w)


def merit_delta_rule_backward(plan, dy, q, k, g, beta, states, *, lens=None, dh_last=None, dh0=False, stream=None):
    """{'dq', 'dk', 'dv', 'dg', 'dbeta', 'dh0'}; dg, dbeta and dh0 in fp32, dg None where there is no g."""
    r = _call(plan, "merit_delta_rule_backward", (dy, q, k, g, beta, states, lens, dh_last) + (None,) * 6,
              0x1700 | (g is not None) << 11 | bool(dh0) << 13, stream)
    return dict(zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), r))


def merit_delta_rule_step(plan, h, q, k, v, g, beta, *, h_out=None, y=None, stream=None):
    """One token more, q, k[B, key_heads, Dk], v[B, heads, Dv], from the state h[B, heads, Dk, Dv]: (y, the state now); h_out
    may be h."""
    return _call(plan, "merit_delta_rule_step", (h, q, k, v, g, beta, y, h_out), 0xC0, stream)


# --------------------------------------------------------------------------
# the norms before and after a block
# --------------------------------------------------------------------------
def merit_plan_block_norm(dtype, B, L, C, *, stream=None, layer=False, eps=1e-6, act=MERIT_ACT_NONE, after=True,
                          before=True) -> TokenPlan:
    """Rows x[B, L, C].  stream: the type of the residual stream (dtype if not given, or MERIT_F32); layer: norms subtract the
    mean; act: of the gate; after, before: which norms there are."""
    b, h = _binding(), ctypes.c_void_p()
    stream = dtype if stream is None else stream
    b._check(b.lib().merit_plan_block_norm(dtype, stream, B, L, C, float(eps), int(bool(layer)), act, int(bool(after)),
                                           int(bool(before)), ctypes.byref(h)), "merit_plan_block_norm")
    x, stat, c = (B, L, C), (B, L), (C,)
    R = _T if stream == dtype else _F32
    plan = TokenPlan(h, dtype, {
        "merit_block_norm": (0, [("x", _T, x, 2, "in"), ("z", _T, x, 2, "opt"), ("r", R, x, 2, "opt"),
                                 ("after_weight", _P, c, 0, "opt"), ("after_bias", _P, c, 0, "opt"), ("scale", _P, c, 0, "opt"),
                                 ("before_weight", _P, c, 0, "opt"), ("before_bias", _P, c, 0, "opt"), ("out", R, x, 2, "out"),
                                 ("n", _T, x, 2, "out?"), ("after_mean", _F32, stat, 0, "out?"), ("after_rstd", _F32, stat, 0, "out?"),
                                 ("before_mean", _F32, stat, 0, "out?"), ("before_rstd", _F32, stat, 0, "out?")]),
        "merit_block_norm_backward": (1, [("dout", R, x, 2, "opt"), ("dn", _T, x, 2, "in" if before else "opt"), ("x", _T, x, 2, "in"),
                                          ("z", _T, x, 2, "opt"), ("r", R, x, 2, "opt"),
                                          ("after_weight", _P, c, 0, "opt"), ("after_bias", _P, c, 0, "opt"),
                                          ("scale", _P, c, 0, "opt"), ("before_weight", _P, c, 0, "opt"),
                                          ("after_mean", _F32, stat, 0, "opt"), ("after_rstd", _F32, stat, 0, "opt"),
                                          ("before_mean", _F32, stat, 0, "opt"), ("before_rstd", _F32, stat, 0, "opt"),
                                          ("dx", _T, x, 2, "out"), ("dz", _T, x, 2, "out?"), ("dr", R, x, 2, "out?"),
                                          ("dafter_weight", _F32, c, 0, "out?"), ("dafter_bias", _F32, c, 0, "out?"),
                                          ("dscale", _F32, c, 0, "out?"), ("dbefore_weight", _F32, c, 0, "out?"),
                                          ("dbefore_bias", _F32, c, 0, "out?")])})
    plan._norms = bool(after), bool(before), bool(layer)
    return plan


def _norms(plan, where):
    plan.operands(where)                # (a plan of another operator is an error here)
    return plan._norms


def merit_block_norm(plan, x, z=None, r=None, *, after_weight=None, after_bias=None, scale=None, before_weight=None,
                     before_bias=None, stats=False, out=None, n=None, stream=None):
    """u = norm(x) after_weight + after_bias, out = r + scale u act(z), n = norm(out) before_weight + before_bias: (out, n),
    n None without the second norm; with stats: and what the backward pass takes.  out may be r."""
    after, before, layer = _norms(plan, "merit_block_norm")
    kept = (stats and after and layer, stats and after, stats and before and layer, stats and before)
    a = _call(plan, "merit_block_norm", (x, z, r, after_weight, after_bias, scale, before_weight, before_bias, out, n) + (None,) * 4,
              0x100 | before << 9 | _bits(*kept) << 10, stream)
    return (a[0], a[1], a[2:]) if stats else a[:2]


def merit_block_norm_backward(plan, dout, dn, x, z, r, stats, *, after_weight=None, after_bias=None, scale=None,
                              before_weight=None, before_bias=None, dr=False, stream=None):
    """{'dx', 'dz', 'dr', 'dafter_weight', 'dafter_bias', 'dscale', 'dbefore_weight', 'dbefore_bias'}: None for an operand that is
    absent.  dout: the gradient of out, or None; dn: that of n; dr (True, or a tensor, which may be dout): the gradient of r."""
    plan.operands("merit_block_norm_backward")
    given = None if isinstance(dr, bool) else dr
    want = _bits(True, z is not None, dr is not False, after_weight is not None, after_bias is not None, scale is not None,
                 before_weight is not None, before_bias is not None)
    a = _call(plan, "merit_block_norm_backward",
              (dout, dn, x, z, r, after_weight, after_bias, scale, before_weight) + tuple(stats) +
              (None, None, given) + (None,) * 5, want << 13, stream)
    return dict(zip(("dx", "dz", "dr", "dafter_weight", "dafter_bias", "dscale", "dbefore_weight", "dbefore_bias"), a))
