"""The gated delta rule and the norms before and after a block, fused with the block's gate and residual scale, as programs
call them: listed() and draw() name the sizes, prepare() makes what a program holds before the call, run() makes the call, in
plain torch operations or (own) through the library.

Kinds of case:
  delta        gated delta rule over a batch of prompts            q, k[B, L, K, Dk], v[B, L, H, Dv], state[B, H, Dk, Dv]
  delta_train  the same with its backward pass
  delta_step   one more token for every sequence, from the kept state
  norm         the end of a block: norm(x) gated, scaled, added to the residual stream, and the norm before the next block
  norm_train   the same with its backward pass
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
CHUNK = 64      # tokens that the plain form takes at once


# --------------------------------------------------------------------------
# sizes
# --------------------------------------------------------------------------
def _delta(kind, dtype, B, L, H, K, Dk, Dv, **more):
    return dict(dict(kind=kind, dtype=dtype, B=B, L=L, H=H, K=K, Dk=Dk, Dv=Dv, unit=True, ragged=False, sliced=False), **more)


def _norm(kind, dtype, B, L, C, **more):
    return dict(dict(kind=kind, dtype=dtype, B=B, L=L, C=C, stream=dtype, layer=False, gate="none", act="none", after=True,
                     scale=False, add=True, before=True, sliced=False), **more)


def listed():
    return [
        # serving: the next token of one sequence, a small model: latency is all of it
        dict(_delta("delta_step", "bf16", 1, 1, 4, 4, 64, 64), name="delta_step_1x4x64x64"),
        # serving: the next token of 32 sequences; the states are 32 MiB, read and written
        dict(_delta("delta_step", "bf16", 32, 1, 16, 8, 128, 128), name="delta_step_32x16x128x128"),
        # a small model in full precision: nothing is a multiple of anything, two prompts of different lengths
        dict(_delta("delta", "f32", 2, 333, 3, 3, 40, 50, ragged=True), name="delta_2x333x3x40x50_f32"),
        # serving: one long prompt of odd length, q, k and v slices of one projection, two value heads to a key head
        dict(_delta("delta", "bf16", 1, 8191, 16, 8, 128, 128, sliced=True), name="delta_1x8191x16x128x128"),
        # training a small model on sequences that no tile divides
        dict(_delta("delta_train", "f16", 3, 1000, 6, 6, 64, 96), name="delta_train_3x1000x6x64x96"),
        # training on 8 x 2048 tokens: the largest
        dict(_delta("delta_train", "bf16", 8, 2048, 16, 16, 128, 128, sliced=True), name="delta_train_8x2048x16x128x128"),
        # serving: a block's end for the next token of 16 sequences: added to the residual stream, normalised for the next block
        dict(_norm("norm", "bf16", 16, 1, 2048, after=False), name="norm_16x1x2048"),
        # scoring 8 x 2048 tokens: norms on both sides of the block, a residual stream in fp32, a scale a channel
        dict(_norm("norm", "bf16", 8, 2048, 2048, stream="f32", scale=True), name="norm_8x2048x2048"),
        # a small model in full precision: layer norms, a gate a sequence, odd sizes
        dict(_norm("norm_train", "f32", 3, 333, 770, layer=True, gate="sequence", scale=True), name="norm_train_3x333x770_f32"),
        # training: the norm of each head's result behind a recurrence, gated by half of a projection; rows of one head
        dict(_norm("norm_train", "bf16", 16384, 16, 128, gate="token", act="silu", add=False, before=False, sliced=True),
             name="norm_train_16384x16x128"),
        # training on 8 x 2048 tokens: both norms, a scale a channel
        dict(_norm("norm_train", "bf16", 8, 2048, 2048, scale=True), name="norm_train_8x2048x2048"),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["delta", "delta", "delta_train", "delta_train", "delta_step", "norm", "norm_train"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    while True:
        if kind.startswith("delta"):
            K = _log(rng, 1, 16)
            H = K * rng.choice([1, 1, 2, 4])
            Dk, Dv = (rng.choice([_log(rng, 8, 128), 64, 128]), rng.choice([_log(rng, 8, 256), 64, 128]))
            if kind == "delta_step":
                c = _delta(kind, dtype, _log(rng, 1, 256), 1, H, K, Dk, Dv)
            else:
                c = _delta(kind, dtype, _log(rng, 1, 32), _log(rng, 1, 16384), H, K, Dk, Dv, ragged=rng.random() < 0.5,
                           sliced=rng.random() < 0.5)
            # (a key of one sign's few values has next to no direction: keys of 8 and more)
            if c["B"] * H * max(c["L"], 64) * Dk * Dv <= (1 << 31 if kind.endswith("_train") else 1 << 32):
                return c
        else:
            rows = _log(rng, 1, 16384)
            L = rng.choice([1, rows, _log(rng, 1, rows)])
            C = rng.choice([_log(rng, 8, 8192), 64 * rng.randint(1, 64)])
            add = rng.random() < 0.8
            gate = rng.choice(["none", "token", "sequence"])
            c = _norm(kind, dtype, max(1, rows // L), L, C, stream=rng.choice([dtype, "f32"]) if add else dtype,
                      layer=rng.random() < 0.3, gate=gate, act=rng.choice(["none", "silu", "sigmoid"]) if gate != "none" else "none",
                      after=rng.random() < 0.7, scale=rng.random() < 0.5, add=add, before=add and rng.random() < 0.8,
                      sliced=rng.random() < 0.3)
            if rows * C <= 1 << 25 and (c["after"] or c["before"]):
                return c


def work(case):
    c, kind = dict(case), case["kind"]
    e = 4 if c["dtype"] == "f32" else 2
    train = kind.endswith("_train")
    if kind.startswith("delta"):
        rows = c["B"] * c["L"]
        qk, v, s = rows * c["K"] * c["Dk"] * e, rows * c["H"] * c["Dv"] * e, rows * c["H"] * 4
        state = c["B"] * c["H"] * c["Dk"] * c["Dv"]
        # a state at one token: the decay, the read along k, the outer product, the read along q; each twice more for its gradients
        flops = rows * c["H"] * c["Dk"] * c["Dv"] * 7 * (3 if train else 1)
        if kind == "delta_step":
            return {"bytes": 2 * qk + 2 * v + 2 * s + 8 * state, "flops": flops}
        return {"bytes": (4 * qk + 4 * v + 4 * s if train else 2 * qk + 2 * v + 2 * s) + 4 * state, "flops": flops}
    n, f = c["B"] * c["L"] * c["C"], 4 if c["stream"] == "f32" else 2 if c["stream"] != "f32" and e == 2 else 4
    z = {"none": 0, "token": n, "sequence": c["B"] * c["C"]}[c["gate"]] * e
    # x, z and the stream in, the stream and the next block's input out; backward: their gradients
    fwd = n * e + z + n * f * (2 if c["add"] else 1) + (n * e if c["before"] else 0)
    back = n * e + (n * e if z else 0) + n * f * (2 if c["add"] else 1) + (n * e if c["before"] else 0)
    vectors = 4 * c["C"] * (c["after"] + c["before"]) * (2 if c["layer"] else 1) + 4 * c["C"] * c["scale"]
    return {"bytes": fwd + (back if train else 0) + vectors * (2 if train else 1), "flops": n * (40 if train else 14)}


# --------------------------------------------------------------------------
# what a program holds before the call
# --------------------------------------------------------------------------
def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    T, f32 = TYPES[c["dtype"]], torch.float32

    def normal(*shape, dtype=T, mean=0.0, std=1.0):
        return torch.randn(shape, generator=g, device=DEVICE).mul_(std).add_(mean).to(dtype)

    def uniform(*shape, lo=0.0, hi=1.0):
        return torch.rand(shape, generator=g, device=DEVICE).mul_(hi - lo).add_(lo)

    s, kind = dict(case=c), c["kind"]
    B, L = c["B"], c["L"]
    if kind.startswith("delta"):
        H, K, Dk, Dv = c["H"], c["K"], c["Dk"], c["Dv"]
        if c["sliced"]:     # one projection gives q, k and v side by side
            side = normal(B, L, 2 * K * Dk + H * Dv)
            q, k, v = side.split([K * Dk, K * Dk, H * Dv], dim=2)
            s["q"], s["k"], s["v"] = q.unflatten(2, (K, Dk)), k.unflatten(2, (K, Dk)), v.unflatten(2, (H, Dv))
        else:
            s["q"], s["k"], s["v"] = normal(B, L, K, Dk), normal(B, L, K, Dk), normal(B, L, H, Dv)
        # decays as learnt ones are: a rate a head, a step a token; most states fade over tens to thousands of tokens
        rate, bias = uniform(H, lo=1.0, hi=16.0), torch.log(torch.expm1(torch.exp(uniform(H, lo=math.log(1e-3), hi=math.log(1e-1)))))
        step = normal(B, L, H, dtype=f32) + bias
        s["g"] = -rate * torch.logaddexp(step, torch.zeros_like(step))
        s["beta"] = torch.sigmoid(normal(B, L, H, dtype=f32))
        s["scale"] = Dk ** -0.5
        if kind == "delta_step":
            for n in ("q", "k", "v", "g", "beta"):
                s[n] = s[n][:, 0]
            s["h"] = normal(B, H, Dk, Dv, dtype=f32, std=Dk ** -0.5)
            s["h_out"] = torch.empty_like(s["h"])
        else:
            s["lens"] = _lengths(B, L, g) if c["ragged"] else None
            if kind == "delta_train":
                s["dy"] = normal(B, L, H, Dv)
    else:
        C, R = c["C"], TYPES[c["stream"]]
        # a block's result: channels of different sizes and means
        x = (normal(B, L, C, dtype=f32) * uniform(C, lo=0.3, hi=3.0) + normal(C, dtype=f32, std=0.3)).to(T)
        s["x"] = torch.cat([x, x[..., :8]], dim=-1)[..., :C] if c["sliced"] else x
        if c["gate"] == "token":    # the second half of a projection
            s["z"] = normal(B, L, 2 * C)[..., C:] if c["sliced"] else normal(B, L, C)
        else:
            s["z"] = normal(B, 1, C).expand(B, L, C) if c["gate"] == "sequence" else None
        s["r"] = normal(B, L, C, dtype=R, std=2.0) if c["add"] else None
        for w, b, on in (("aw", "ab", c["after"]), ("bw", "bb", c["before"])):
            s[w] = normal(C, dtype=f32, mean=1.0, std=0.2) if on else None
            s[b] = normal(C, dtype=f32, std=0.2) if on and c["layer"] else None
        s["scale"] = uniform(C, lo=0.05, hi=0.5) if c["scale"] else None
        if kind == "norm_train":
            s["dout"] = normal(B, L, C, dtype=R) if c["add"] or not c["before"] else None
            s["dn"] = normal(B, L, C) if c["before"] else None
    if own:     # the plan that a program makes once for its sizes
        s["plan"] = _plan(c)
    return s


def _lengths(B, L, g):
    """Lengths of B prompts: the first is the longest, the others anything from 1 on."""
    n = torch.randint(1, L + 1, (B,), generator=g, device=DEVICE, dtype=torch.int32)
    n[0] = L
    return n


def _plan(c):
    from paper_1911_03458_amd import binding as mb
    code = {"bf16": mb.MERIT_BF16, "f16": mb.MERIT_F16, "f32": mb.MERIT_F32}
    if c["kind"].startswith("delta"):
        return mb.merit_plan_delta_rule(code[c["dtype"]], c["B"], c["L"], c["H"], c["K"], c["Dk"], c["Dv"], normalize=c["unit"])
    act = {"none": mb.MERIT_ACT_NONE, "silu": mb.MERIT_ACT_SILU, "sigmoid": mb.MERIT_ACT_SIGMOID}[c["act"]]
    return mb.merit_plan_block_norm(code[c["dtype"]], c["B"], c["L"], c["C"], stream=code[c["stream"]], layer=c["layer"], eps=EPS,
                                    act=act, after=c["after"], before=c["before"])


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_1911_03458_amd import binding as mb
    kind, plan = s["case"]["kind"], s["plan"]
    if kind == "delta":
        y, h = mb.merit_delta_rule(plan, s["q"], s["k"], s["v"], s["g"], s["beta"], lens=s["lens"], final=True)
        return {"y": y, "h": h}
    if kind == "delta_step":
        y, h = mb.merit_delta_rule_step(plan, s["h"], s["q"], s["k"], s["v"], s["g"], s["beta"], h_out=s["h_out"])
        return {"y": y, "h": h}
    if kind == "delta_train":
        y, h, states = mb.merit_delta_rule(plan, s["q"], s["k"], s["v"], s["g"], s["beta"], lens=s["lens"], final=True, states=True)
        d = mb.merit_delta_rule_backward(plan, s["dy"], s["q"], s["k"], s["g"], s["beta"], states, lens=s["lens"])
        return {"y": y, "h": h, **{k: d[k] for k in ("dq", "dk", "dv", "dg", "dbeta")}}
    vectors = dict(after_weight=s["aw"], after_bias=s["ab"], scale=s["scale"], before_weight=s["bw"], before_bias=s["bb"])
    if kind == "norm":
        out, n = mb.merit_block_norm(plan, s["x"], s["z"], s["r"], **vectors)
        return {"out": out, "n": n}
    out, n, stats = mb.merit_block_norm(plan, s["x"], s["z"], s["r"], stats=True, **vectors)
    d = mb.merit_block_norm_backward(plan, s["dout"], s["dn"], s["x"], s["z"], s["r"], stats, dr=s["r"] is not None, **vectors)
    return {"out": out, "n": n, **d}


def _run_plain(s):
    kind = s["case"]["kind"]
    return _norm_plain(s) if kind.startswith("norm") else _step_plain(s) if kind == "delta_step" else _delta_plain(s)


def _unit(x):
    return x * torch.rsqrt((x * x).sum(-1, keepdim=True) + EPS)


def _unit_grad(d, x):
    """The gradient of x through _unit."""
    r = torch.rsqrt((x * x).sum(-1, keepdim=True) + EPS)
    u = x * r
    return r * (d - u * (u * d).sum(-1, keepdim=True))


def _step_plain(s):
    c, T = s["case"], s["v"].dtype
    each = c["H"] // c["K"]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if c["unit"]:
        q, k = _unit(q), _unit(k)
    q, k = q.repeat_interleave(each, dim=1), k.repeat_interleave(each, dim=1)
    h = s["h"] * torch.exp(s["g"])[..., None, None]
    u = s["beta"].float()[..., None] * (v - (h * k[..., None]).sum(-2))
    h = h + k[..., None] * u[..., None, :]
    s["h_out"].copy_(h)
    return {"y": ((h * q[..., None]).sum(-2) * s["scale"]).to(T), "h": s["h_out"]}


def _t(x):
    return x.transpose(-1, -2).contiguous()


def _delta_plain(s):
    """Chunks of CHUNK tokens: what a chunk's tokens add to the state together solves a triangular system."""
    c, T = s["case"], s["v"].dtype
    B, L, H, K, Dk, Dv = (c[n] for n in ("B", "L", "H", "K", "Dk", "Dv"))
    train = c["kind"] == "delta_train"
    n, each = -(-L // CHUNK), H // K
    lens = s["lens"]
    inside = torch.ones(B, L, dtype=torch.bool, device=s["v"].device) if lens is None else \
        torch.arange(L, device=s["v"].device)[None] < lens[:, None]

    def chunks(x):      # [B, L, H, ...] -> [B, H, n, CHUNK, ...], zeros behind a sequence's end
        x = x.masked_fill(~inside.view(B, L, *[1] * (x.dim() - 2)), 0.0)
        x = torch.cat([x, x.new_zeros(B, n * CHUNK - L, *x.shape[2:])], dim=1)
        return x.unflatten(1, (n, CHUNK)).movedim(3, 1).contiguous()

    def tokens(x):      # back: [B, H, n, CHUNK, ...] -> [B, L, H, ...]
        return x.movedim(1, 3).flatten(1, 2)[:, :L].contiguous()

    raw_q, raw_k = s["q"].float(), s["k"].float()
    q, k = (_unit(raw_q), _unit(raw_k)) if c["unit"] else (raw_q, raw_k)
    q = chunks(q.repeat_interleave(each, dim=2)) * s["scale"]
    k, v = chunks(k.repeat_interleave(each, dim=2)), chunks(s["v"].float())
    beta, g = chunks(s["beta"].float())[..., None], chunks(s["g"].double())
    # decays between two tokens of a chunk: differences of long sums, in 64 bits
    G = g.cumsum(-1)
    lower = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=G.device).tril()
    fade = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~lower, -math.inf)).float()
    strict = fade.masked_fill(torch.eye(CHUNK, dtype=torch.bool, device=G.device), 0.0)
    into, rest = torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None]
    whole = torch.exp(G[..., -1]).float()[..., None, None]
    # (1 + A) u = beta (v - into k S): the inverse of a triangular matrix, as a product of powers of it, in 64 bits
    A = beta * strict * (k @ _t(k))
    eye, X = torch.eye(CHUNK, dtype=torch.float64, device=G.device), -A.double()
    inv = eye + X
    m = 2
    while m < CHUNK:
        X = X @ X
        inv = inv + inv @ X
        m *= 2
    inv = inv.float()
    P = fade * (q @ _t(k))
    S = k.new_zeros(B, H, Dk, Dv)
    before, us, deltas = [], [], []
    for i in range(n):
        before.append(S)
        d = v[:, :, i] - into[:, :, i] * (k[:, :, i] @ S)
        u = inv[:, :, i] @ (beta[:, :, i] * d)
        S = whole[:, :, i] * S + _t(k[:, :, i]) @ (rest[:, :, i] * u)
        us.append(u)
        deltas.append(d)
    S0, u, d = torch.stack(before, 2), torch.stack(us, 2), torch.stack(deltas, 2)
    y = tokens(into * (q @ S0) + P @ u).to(T)
    if not train:
        return {"y": y, "h": S}
    dy = chunks(s["dy"].float())
    dS = torch.zeros_like(S)
    Pt, invt, kt, qt = _t(P), _t(inv), _t(k), _t(q)
    behind, dxs = [], []
    for i in reversed(range(n)):
        behind.append(dS)
        dx = invt[:, :, i] @ (Pt[:, :, i] @ dy[:, :, i] + rest[:, :, i] * (k[:, :, i] @ dS))
        dS = whole[:, :, i] * dS + qt[:, :, i] @ (into[:, :, i] * dy[:, :, i]) - kt[:, :, i] @ (into[:, :, i] * beta[:, :, i] * dx)
        dxs.append(dx)
    dS, dx = torch.stack(behind[::-1], 2), torch.stack(dxs[::-1], 2)
    dv = beta * dx
    S0t, ut = _t(S0), _t(u)
    dP, dA = fade * (dy @ ut), -strict * (dx @ ut) * beta
    dq = into * (dy @ S0t) + dP @ k
    rows = dA @ k - into * (dv @ S0t)                           # of k as the token that reads
    cols_S = rest * (u @ _t(dS))
    cols = _t(dP) @ q + _t(dA) @ k + cols_S                     # of k as the token that was written
    # a token's own strength: what it would have added at strength one is what it adds where A is not in the way
    held = d - strict * (k @ _t(k)) @ u
    dbeta = (dx * held).sum(-1)
    dG = (q * dq).double().sum(-1) + (k * (rows - cols)).double().sum(-1)
    dG[..., -1] += (whole * S0 * dS).double().sum((-1, -2)) + (k * cols_S).double().sum((-1, -2))
    dg = dG.flip(-1).cumsum(-1).flip(-1).float()

    def keys(x):        # the heads that share a key head
        return tokens(x).unflatten(2, (K, each)).sum(3)

    dq, dk = keys(dq) * s["scale"], keys(rows + cols)
    if c["unit"]:
        dq, dk = _unit_grad(dq, raw_q), _unit_grad(dk, raw_k)
    hide = ~inside[:, :, None]
    return {"y": y, "h": S, "dq": dq.masked_fill(hide[..., None], 0.0).to(T), "dk": dk.masked_fill(hide[..., None], 0.0).to(T),
            "dv": tokens(dv).masked_fill(hide[..., None], 0.0).to(T), "dg": tokens(dg).masked_fill(hide, 0.0),
            "dbeta": tokens(dbeta).masked_fill(hide, 0.0)}


def _gate(z, act):
    return z if act == "none" else torch.sigmoid(z) * (z if act == "silu" else 1.0)


def _gate_slope(z, act):
    q = torch.sigmoid(z)
    return torch.ones_like(z) if act == "none" else q * (1 - q) if act == "sigmoid" else q * (1 + z * (1 - q))


def _normed(x, layer):
    """(x less its mean over its root mean square, one over that) along the channels; without a layer norm the mean stays."""
    d = x - x.mean(-1, keepdim=True) if layer else x
    r = torch.rsqrt((d * d).mean(-1, keepdim=True) + EPS)
    return d * r, r


def _normed_grad(dw, xh, r, layer):
    return r * (dw - (dw.mean(-1, keepdim=True) if layer else 0.0) - xh * (dw * xh).mean(-1, keepdim=True))


def _norm_plain(s):
    c, x, T, R = s["case"], s["x"].float(), s["x"].dtype, TYPES[s["case"]["stream"]]
    one, none = x.new_ones(c["C"]), x.new_zeros(c["C"])
    aw, bw, scale = (one if s[k] is None else s[k] for k in ("aw", "bw", "scale"))
    ab, bb = (none if s[k] is None else s[k] for k in ("ab", "bb"))
    xh, rx = _normed(x, c["layer"]) if c["after"] else (x, None)
    u = xh * aw + ab
    z = None if s["z"] is None else s["z"].float()
    e = None if z is None else _gate(z, c["act"])
    t = u if z is None else u * e
    o = scale * t if s["r"] is None else s["r"].float() + scale * t
    out = {"out": o.to(R), "n": None}
    if c["before"]:
        oh, ro = _normed(o, c["layer"])
        out["n"] = (oh * bw + bb).to(T)
    if c["kind"] == "norm":
        return out
    do = x.new_zeros(x.shape) if s["dout"] is None else s["dout"].float()
    if c["before"]:
        dn = s["dn"].float()
        do = do + _normed_grad(dn * bw, oh, ro, c["layer"])
        out["dbefore_weight"] = (dn * oh).sum((0, 1))
        out["dbefore_bias"] = dn.sum((0, 1)) if c["layer"] else None
    if s["r"] is not None:
        out["dr"] = do.to(R)
    if c["scale"]:
        out["dscale"] = (do * t).sum((0, 1))
    dt = do * scale
    du = dt if z is None else dt * e
    if z is not None:
        out["dz"] = (dt * u * _gate_slope(z, c["act"])).to(T)
    if c["after"]:
        out["dafter_weight"] = (du * xh).sum((0, 1))
        out["dafter_bias"] = du.sum((0, 1)) if c["layer"] else None
        du = _normed_grad(du * aw, xh, rx, c["layer"])
    out["dx"] = du.to(T)
    return out


# --------------------------------------------------------------------------
# the definitions in 64 bits, token by token
# --------------------------------------------------------------------------
def exact(case, seed):
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in prepare(case, seed).items()}
    f = _norm_exact if case["kind"].startswith("norm") else _delta_exact
    with torch.no_grad():
        return {k: None if v is None else np.array(v.cpu().numpy()) for k, v in f(s, s["case"]).items()}


def _delta_exact(s, c):
    B, L, H, K, Dk, Dv = (c[n] for n in ("B", "L", "H", "K", "Dk", "Dv"))
    kind, dev = c["kind"], s["v"].device
    head = torch.arange(H, device=dev) // (H // K)
    one = kind == "delta_step"
    q, k, v, a, b = (s[n][:, None] if one else s[n] for n in ("q", "k", "v", "g", "beta"))
    lq, lk = (torch.sqrt(x.square().sum(-1, keepdim=True) + EPS) if c["unit"] else torch.ones_like(x[..., :1]) for x in (q, k))
    qh, kh = (q / lq)[:, :, head] * s["scale"], (k / lk)[:, :, head]
    a = torch.exp(a)
    lens = torch.full((B,), L, device=dev) if s.get("lens") is None else s["lens"].long()
    live = (torch.arange(L, device=dev)[None] < lens[:, None]).double()     # behind the end: no decay, nothing comes in
    S = s["h"] if one else v.new_zeros(B, H, Dk, Dv)
    y = torch.zeros_like(v)
    kept = v.new_empty(L + 1, B, H, Dk, Dv) if kind == "delta_train" else None
    for t in range(L):
        if kept is not None:
            kept[t] = S
        on = live[:, t, None, None, None]
        faded = S * (a[:, t, :, None, None] * on + (1 - on))
        miss = v[:, t] - torch.einsum("bhkv,bhk->bhv", faded, kh[:, t])
        S = faded + on * torch.einsum("bhk,bhv->bhkv", kh[:, t], miss * b[:, t, :, None])
        y[:, t] = torch.einsum("bhkv,bhk->bhv", S, qh[:, t]) * live[:, t, None, None]
    if one:
        return {"y": y[:, 0], "h": S}
    out = {"y": y, "h": S}
    if kind != "delta_train":
        return out
    kept[L] = S
    D = torch.zeros_like(S)                     # the gradient of the state behind token t
    dq, dk, dv = torch.zeros_like(qh), torch.zeros_like(kh), torch.zeros_like(v)
    dg, db = torch.zeros_like(a), torch.zeros_like(b)
    for t in range(L - 1, -1, -1):
        on = live[:, t, None, None]
        dy = s["dy"][:, t] * on
        dq[:, t] = torch.einsum("bhkv,bhv->bhk", kept[t + 1], dy)
        D = D + torch.einsum("bhk,bhv->bhkv", qh[:, t], dy)
        decay = a[:, t, :, None, None]
        faded = kept[t] * decay
        miss = v[:, t] - torch.einsum("bhkv,bhk->bhv", faded, kh[:, t])
        along = torch.einsum("bhkv,bhk->bhv", D, kh[:, t])
        db[:, t] = (along * miss).sum(-1) * live[:, t, None]
        dmiss = along * b[:, t, :, None]
        dv[:, t] = dmiss * on
        dk[:, t] = (torch.einsum("bhkv,bhv->bhk", D, miss * b[:, t, :, None]) - torch.einsum("bhkv,bhv->bhk", faded, dmiss)) * on
        back = D - torch.einsum("bhk,bhv->bhkv", kh[:, t], dmiss)
        dg[:, t] = (back * faded).sum((-1, -2)) * live[:, t, None]
        D = torch.where(on[..., None] > 0, back * decay, D)

    def through(d, x, length):                  # the sum over the heads of a key head, through the division by the length
        d = d.view(B, L, K, H // K, Dk).sum(3)
        return d / length - (x * (x * d).sum(-1, keepdim=True) / length ** 3 if c["unit"] else 0.0)

    return {**out, "dq": through(dq, q, lq) * s["scale"], "dk": through(dk, k, lk), "dv": dv, "dg": dg, "dbeta": db}


def _norm_exact(s, c):
    C, x, z = c["C"], s["x"], s["z"]
    tanh = torch.tanh
    shift = (lambda v: v - v.sum(-1, keepdim=True) / C) if c["layer"] else (lambda v: v)

    def length(v):
        return torch.sqrt(v.pow(2).sum(-1, keepdim=True) / C + EPS)

    def affine(v, w, b):
        v = v if w is None else v * w
        return v if b is None else v + b

    half = None if z is None else 0.5 * (1 + tanh(z / 2))      # the logistic function
    e = {"none": z, "silu": None if z is None else z * half, "sigmoid": half}[c["act"]]
    xc = shift(x) if c["after"] else x
    xl = length(xc) if c["after"] else 1.0
    u = affine(xc / xl, s["aw"], s["ab"])
    t = u if z is None else e * u
    o = t if s["scale"] is None else t * s["scale"]
    o = o if s["r"] is None else o + s["r"]
    res = {"out": o, "n": None}
    if c["before"]:
        oc = shift(o)
        ol = length(oc)
        res["n"] = affine(oc / ol, s["bw"], s["bb"])
    if c["kind"] == "norm":
        return res

    def back(d, vc, l):     # through v -> shift(v) / length
        d = d / l - vc * (d * vc).sum(-1, keepdim=True) / (C * l ** 3)
        return shift(d)

    do = torch.zeros_like(x) if s["dout"] is None else s["dout"].clone()
    if c["before"]:
        do += back(s["dn"] * s["bw"], oc, ol)
        res["dbefore_weight"] = torch.einsum("blc,blc->c", s["dn"], oc / ol)
        res["dbefore_bias"] = s["dn"].sum((0, 1)) if c["layer"] else None
    if s["r"] is not None:
        res["dr"] = do
    if s["scale"] is not None:
        res["dscale"] = torch.einsum("blc,blc->c", do, t)
        do = do * s["scale"]
    if z is not None:
        slope = {"none": 1.0, "sigmoid": half * (1 - half), "silu": half + z * half * (1 - half)}[c["act"]]
        res["dz"] = do * u * slope
        do = do * e
    if c["after"]:
        res["dafter_weight"] = torch.einsum("blc,blc->c", do, xc / xl)
        res["dafter_bias"] = do.sum((0, 1)) if c["layer"] else None
        do = back(do * s["aw"], xc, xl)
    res["dx"] = do
    return res
