"""The operators along a sequence of tokens -- short causal convolution, selective state space scan, group norm with an
activation, all channels last -- as programs call them: listed() and draw() name the sizes, prepare() makes what a program
holds before the call, run() makes the call, in plain torch operations or (own) through the library.

Kinds of case:
  norm        group norm + activation of a layer's output          x[N, S, C], S positions share the statistics
  norm_train  the same with its backward pass
  conv        short causal convolution over a batch of prompts     x[B, L, D], window of K tokens
  conv_train  the same with its backward pass
  conv_step   one more token for every sequence, from the kept K - 1 tokens
  scan        selective scan over a batch of prompts               x[B, L, D], state[B, D, N]
  scan_train  the same with its backward pass
  scan_step   one more token for every sequence, from the kept state
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# --------------------------------------------------------------------------
# sizes
# --------------------------------------------------------------------------
def listed():
    return [
        # the norm of 16 sequences' next token, heads of 64 channels: latency is all of it
        dict(name="norm_16x1x1024", kind="norm", dtype="f16", N=16, S=1, C=1024, G=16, act="none"),
        # the output of a 256-channel convolution layer on 8 images
        dict(name="norm_8x3136x256", kind="norm", dtype="bf16", N=8, S=3136, C=256, G=32, act="silu"),
        # training on a first block's large maps, few channels
        dict(name="norm_train_16x12544x64", kind="norm_train", dtype="f16", N=16, S=12544, C=64, G=8, act="silu"),
        # training a token mixer: every token of 8 x 2048 has its own statistics, heads of 128 channels
        dict(name="norm_train_16384x1x2048", kind="norm_train", dtype="bf16", N=16384, S=1, C=2048, G=16, act="silu"),
        # serving: the next token of 32 sequences
        dict(name="conv_step_32x2048", kind="conv_step", dtype="bf16", B=32, D=2048, K=4, act="silu"),
        # serving: three prompts of different lengths, padded to the longest, the convolution's input half of a projection
        dict(name="conv_3x4099x1536", kind="conv", dtype="bf16", B=3, L=4099, D=1536, K=4, act="silu", ragged=True,
             sliced=True),
        # training on 8 x 2048 tokens
        dict(name="conv_train_8x2048x2048", kind="conv_train", dtype="bf16", B=8, L=2048, D=2048, K=4, act="silu",
             sliced=True),
        # serving: the next token of 32 sequences
        dict(name="scan_step_32x2048", kind="scan_step", dtype="bf16", B=32, D=2048, N=16, G=1),
        # serving: one long prompt of odd length; few rows, so the length has to be split
        dict(name="scan_1x8191x2048", kind="scan", dtype="bf16", B=1, L=8191, D=2048, N=16, G=1, gate=True, ragged=False,
             sliced=True),
        # a small model in full precision: nothing is a multiple of anything, two prompts of different lengths
        dict(name="scan_2x333x90_f32", kind="scan", dtype="f32", B=2, L=333, D=90, N=5, G=2, gate=True, ragged=True,
             sliced=False),
        # scoring a batch of 8 x 2048 tokens
        dict(name="scan_8x2048x2048", kind="scan", dtype="bf16", B=8, L=2048, D=2048, N=16, G=1, gate=True, ragged=False,
             sliced=True),
        # training on it: the largest
        dict(name="scan_train_8x2048x2048", kind="scan_train", dtype="bf16", B=8, L=2048, D=2048, N=16, G=1, gate=True,
             sliced=True),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "conv", "conv_train", "conv_step", "scan", "scan", "scan_train", "scan_step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    # (the clipped activation's slope jumps at 0, where two right answers may differ: forward only)
    act = rng.choice(["none", "silu", "silu"] if kind.endswith("_train") else ["none", "relu", "silu"])
    while True:
        if kind.startswith("norm"):
            G = rng.choice([1, 4, 8, 16, 32])
            per = rng.choice([_log(rng, 1, 128), 8 * _log(rng, 1, 16)])
            tokens = rng.random() < 0.5
            N, S = (_log(rng, 1, 16384), 1) if tokens else (_log(rng, 1, 32), _log(rng, 2, 12544))
            # (fewer than 8 values have next to no gradient: what is left of it is rounding)
            if N * S * G * per <= 1 << 25 and S * per >= 8:
                return dict(kind=kind, dtype=dtype, N=N, S=S, C=G * per, G=G, act=act)
        elif kind.startswith("conv"):
            D, K = rng.choice([_log(rng, 8, 2560), 64 * rng.randint(1, 40)]), rng.choice([2, 3, 4, 4, 4])
            if kind == "conv_step":
                return dict(kind=kind, dtype=dtype, B=_log(rng, 1, 256), D=D, K=K, act=act)
            B, L = _log(rng, 1, 32), _log(rng, 1, 16384)
            if B * L * D <= 1 << 25:
                more = dict(ragged=rng.random() < 0.5) if kind == "conv" else {}
                return dict(kind=kind, dtype=dtype, B=B, L=L, D=D, K=K, act=act, sliced=rng.random() < 0.5, **more)
        else:
            G = rng.choice([1, 1, 1, 2, 4])
            D, N = G * rng.choice([_log(rng, 4, 640), 16 * rng.randint(1, 40)]), rng.choice([16, 16, 16, 8, 32, _log(rng, 1, 64)])
            if kind == "scan_step":
                return dict(kind=kind, dtype=dtype, B=_log(rng, 1, 256), D=D, N=N, G=G)
            B, L = _log(rng, 1, 32), _log(rng, 1, 16384)
            if B * L * D * N <= 1 << 29:
                more = dict(ragged=rng.random() < 0.5) if kind == "scan" else {}
                return dict(kind=kind, dtype=dtype, B=B, L=L, D=D, N=N, G=G, gate=rng.random() < 0.7,
                            sliced=rng.random() < 0.5, **more)


def work(case):
    c = dict(case)
    e, kind = (4 if c["dtype"] == "f32" else 2), c["kind"]
    train = kind.endswith("_train")
    if kind.startswith("norm"):
        n = c["N"] * c["S"] * c["C"]
        # forward: x in, y out; backward: dy in, dx out besides (x counts once), dw and db out
        return {"bytes": n * e * (4 if train else 2) + 4 * c["C"] * (4 if train else 2), "flops": n * (28 if train else 8)}
    if kind.startswith("conv"):
        taps = c["D"] * (c["K"] + 1) * 4
        kept = c["B"] * (c["K"] - 1) * c["D"] * e
        if kind == "conv_step":
            n = c["B"] * c["D"]
            return {"bytes": 2 * n * e + 2 * kept + taps, "flops": n * (2 * c["K"] + 4)}
        n = c["B"] * c["L"] * c["D"]
        return {"bytes": n * e * (4 if train else 2) + taps * (2 if train else 1) + kept,
                "flops": n * (2 * c["K"] + 4) * (4 if train else 1)}
    rows = c["B"] * c.get("L", 1)
    n, bc, state = rows * c["D"], rows * c["G"] * c["N"], c["B"] * c["D"] * c["N"] * 4
    params = c["D"] * (c["N"] + 2) * 4
    gate = c.get("gate", True)
    # a state of one channel at one token: an exponential, its argument, the input's and the decay's products, the sum, the read
    flops = n * c["N"] * (26 if train else 7)
    if kind == "scan_step":
        return {"bytes": 4 * n * e + 2 * bc * e + 2 * state + params, "flops": flops}
    if train:   # x, dt, dy, z in, y, dx, ddt, dz out; B, C in, dB, dC out
        return {"bytes": n * e * (8 if gate else 6) + 4 * bc * e + 2 * params + 2 * state, "flops": flops}
    return {"bytes": n * e * (4 if gate else 3) + 2 * bc * e + params + state, "flops": flops}


# --------------------------------------------------------------------------
# what a program holds before the call
# --------------------------------------------------------------------------
def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, f32 = TYPES[c["dtype"]], torch.float32

    def normal(*shape, dtype=T, mean=0.0, std=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(std).add_(mean).to(dtype)

    def uniform(*shape, lo=0.0, hi=1.0):
        return torch.rand(shape, generator=g, device="cuda").mul_(hi - lo).add_(lo)

    s, kind = dict(case=c), c["kind"]
    if kind.startswith("norm"):
        N, S, C = c["N"], c["S"], c["C"]
        # channels of different means and sizes, as a layer's output has them
        s["x"] = (normal(N, S, C, dtype=f32) * uniform(C, lo=0.3, hi=3.0) + normal(C, dtype=f32)).to(T)
        s["weight"], s["bias"] = normal(C, dtype=f32, mean=1.0, std=0.2), normal(C, dtype=f32, std=0.2)
        if kind == "norm_train":
            s["dy"] = normal(N, S, C)
    elif kind.startswith("conv"):
        B, D, K, L = c["B"], c["D"], c["K"], c.get("L", 1)
        # a projection's output, of which the convolution takes the first half of the channels
        s["x"] = normal(B, L, 2 * D)[:, :, :D] if c.get("sliced") else normal(B, L, D)
        s["weight"], s["bias"] = normal(D, K, std=K ** -0.5), normal(D, std=0.2)
        if kind == "conv_step":
            s["x"], s["kept"] = s["x"][:, 0], normal(B, K - 1, D)
            s["kept_out"] = torch.empty_like(s["kept"])
        elif kind == "conv_train":
            s["dy"] = normal(B, L, D)
        else:
            s["lens"] = _lengths(B, L, g) if c["ragged"] else None
    else:
        B, D, N, G, L = c["B"], c["D"], c["N"], c["G"], c.get("L", 1)
        gate = c.get("gate", True)
        s["x"] = normal(B, L, D)
        s["z"] = (normal(B, L, 2 * D)[:, :, D:] if c.get("sliced") else normal(B, L, D)) if gate else None
        s["dt"] = normal(B, L, D, std=0.5)
        # one projection gives a low-rank step, B and C side by side
        if c.get("sliced"):
            side = normal(B, L, 24 + 2 * G * N)[:, :, 24:]
            s["B"], s["C"] = (v.unflatten(2, (G, N)) for v in side.split(G * N, dim=2))
        else:
            s["B"], s["C"] = normal(B, L, G, N), normal(B, L, G, N)
        # decays -1 ... -N, spread a little; steps of 0.001 to 0.1
        s["A"] = -(torch.arange(1, N + 1, device="cuda", dtype=f32) * torch.exp(normal(D, N, dtype=f32, std=0.1)))
        s["skip"] = normal(D, dtype=f32, mean=1.0, std=0.1)
        step = torch.exp(uniform(D, lo=math.log(1e-3), hi=math.log(1e-1)))
        s["dt_bias"] = torch.log(torch.expm1(step))
        if kind == "scan_step":
            for k in ("x", "z", "dt", "B", "C"):
                s[k] = s[k][:, 0]
            s["h"] = normal(B, D, N, dtype=f32)
            s["h_out"] = torch.empty_like(s["h"])
        elif kind == "scan_train":
            s["dy"] = normal(B, L, D)
        else:
            s["lens"] = _lengths(B, L, g) if c["ragged"] else None
    if own:     # the plan that a program makes once for its sizes
        s["plan"] = _plan(c)
    return s


def _lengths(B, L, g):
    """Lengths of B prompts: the first is the longest, the others anything from 1 on."""
    n = torch.randint(1, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    n[0] = L
    return n


def _plan(c):
    from paper_1911_03458_amd import binding as mb
    T = {"bf16": mb.MERIT_BF16, "f16": mb.MERIT_F16, "f32": mb.MERIT_F32}[c["dtype"]]
    act = {"none": mb.MERIT_ACT_NONE, "relu": mb.MERIT_ACT_RELU, "silu": mb.MERIT_ACT_SILU}[c.get("act", "none")]
    if c["kind"].startswith("norm"):
        return mb.merit_plan_group_norm(T, c["N"], c["S"], c["C"], c["G"], 1e-5, act)
    if c["kind"].startswith("conv"):
        return mb.merit_plan_causal_conv(T, c["B"], c.get("L", 1), c["D"], c["K"], act)
    return mb.merit_plan_scan(T, c["B"], c.get("L", 1), c["D"], c["N"], c["G"], True)


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_1911_03458_amd import binding as mb
    kind, plan = s["case"]["kind"], s["plan"]
    if kind == "norm":
        return {"y": mb.merit_group_norm(plan, s["x"], s["weight"], s["bias"])}
    if kind == "norm_train":
        y, mean, rstd = mb.merit_group_norm(plan, s["x"], s["weight"], s["bias"], stats=True)
        dx, dw, db = mb.merit_group_norm_backward(plan, s["dy"], s["x"], mean, rstd, s["weight"], s["bias"])
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    if kind == "conv":
        y, final = mb.merit_causal_conv(plan, s["x"], s["weight"], s["bias"], lens=s["lens"], final=True)
        return {"y": y, "final": final}
    if kind == "conv_train":
        y = mb.merit_causal_conv(plan, s["x"], s["weight"], s["bias"])
        dx, dw, db = mb.merit_causal_conv_backward(plan, s["dy"], s["x"], s["weight"], s["bias"])
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    if kind == "conv_step":
        y, kept = mb.merit_causal_conv_step(plan, s["kept"], s["x"], s["weight"], s["bias"], kept_out=s["kept_out"])
        return {"y": y, "kept": kept}
    if kind == "scan":
        y, h = mb.merit_scan(plan, s["x"], s["dt"], s["A"], s["B"], s["C"], skip=s["skip"], z=s["z"],
                             dt_bias=s["dt_bias"], lens=s["lens"], final=True)
        return {"y": y, "h": h}
    if kind == "scan_step":
        y, h = mb.merit_scan_step(plan, s["h"], s["x"], s["dt"], s["A"], s["B"], s["C"], skip=s["skip"], z=s["z"],
                                  dt_bias=s["dt_bias"], h_out=s["h_out"])
        return {"y": y, "h": h}
    y, h, states = mb.merit_scan(plan, s["x"], s["dt"], s["A"], s["B"], s["C"], skip=s["skip"], z=s["z"],
                                 dt_bias=s["dt_bias"], final=True, states=True)
    grads = mb.merit_scan_backward(plan, s["dy"], s["x"], s["dt"], s["A"], s["B"], s["C"], states, skip=s["skip"], z=s["z"],
                                   dt_bias=s["dt_bias"])
    return {"y": y, "h": h, **{k: v for k, v in grads.items() if v is not None}}


def _act(u, act):
    return u if act == "none" else torch.relu(u) if act == "relu" else u * torch.sigmoid(u)


def _slope(u, act):
    """The activation's derivative (0 at the corner of the clipped one)."""
    if act == "silu":
        q = torch.sigmoid(u)
        return q * (1 + u * (1 - q))
    return (u > 0).float() if act == "relu" else torch.ones_like(u)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind.startswith("norm"):
        return _norm_plain(s)
    if kind.startswith("conv"):
        return _conv_plain(s)
    return _scan_plain(s)


def _norm_plain(s):
    c, x, T = s["case"], s["x"].float(), s["x"].dtype
    N, S, C, G = c["N"], c["S"], c["C"], c["G"]
    w, b = s["weight"], s["bias"]
    v = x.view(N, S, G, C // G)
    d = v - v.mean((1, 3), keepdim=True)
    rstd = torch.rsqrt(d.square().mean((1, 3), keepdim=True) + 1e-5)
    xh = (d * rstd).view(N, S, C)
    u = xh * w + b
    y = _act(u, c["act"]).to(T)
    if c["kind"] == "norm":
        return {"y": y}
    du = s["dy"].float() * _slope(u, c["act"])
    gw, xg = (du * w).view(N, S, G, C // G), xh.view(N, S, G, C // G)
    dx = rstd * (gw - gw.mean((1, 3), keepdim=True) - xg * (gw * xg).mean((1, 3), keepdim=True))
    return {"y": y, "dx": dx.view(N, S, C).to(T), "dw": (du * xh).sum((0, 1)), "db": du.sum((0, 1))}


def _conv_plain(s):
    c, T = s["case"], s["x"].dtype
    B, L, D, K = c["B"], c.get("L", 1), c["D"], c["K"]
    x, w, b = s["x"].float(), s["weight"].float(), s["bias"].float()
    if c["kind"] == "conv_step":
        rows = torch.cat([s["kept"].float(), x[:, None]], dim=1)
        y = _act((rows * w.t()).sum(1) + b, c["act"]).to(T)
        s["kept_out"].copy_(rows[:, 1:])
        return {"y": y, "kept": s["kept_out"]}
    padded = torch.cat([x.new_zeros(B, K - 1, D), x], dim=1)
    u = (padded.unfold(1, K, 1) * w).sum(-1) + b
    y = _act(u, c["act"])
    if c["kind"] == "conv":
        lens = s["lens"]
        n = torch.full((B,), L, device=x.device) if lens is None else lens.long()
        inside = torch.arange(L, device=x.device)[None] < n[:, None]
        last = n[:, None] + torch.arange(K - 1, device=x.device)
        final = padded.gather(1, last[:, :, None].expand(-1, -1, D))
        return {"y": (y * inside[:, :, None]).to(T), "final": final.to(T)}
    du = s["dy"].float() * _slope(u, c["act"])
    later = torch.cat([du, du.new_zeros(B, K - 1, D)], dim=1)
    dx = (later.unfold(1, K, 1) * w.flip(1)).sum(-1)
    dw = (padded.unfold(1, K, 1) * du[..., None]).sum((0, 1))
    return {"y": y.to(T), "dx": dx.to(T), "dw": dw, "db": du.sum((0, 1))}


def _recur(a, b):
    """h[t] = a[t] h[t-1] + b[t] along dimension 1, h[-1] = 0: neighbours are joined in pairs, then the pairs, and so on."""
    n = a.shape[1]
    if n == 1:
        return b
    m = n // 2 * 2
    a0, a1, b0, b1 = a[:, 0:m:2], a[:, 1:m:2], b[:, 0:m:2], b[:, 1:m:2]
    odd = _recur(a0 * a1, a1 * b0 + b1)
    h = torch.empty_like(b)
    h[:, 0], h[:, 1:m:2] = b[:, 0], odd
    h[:, 2::2] = a[:, 2::2] * odd[:, :(n - 1) // 2] + b[:, 2::2]
    return h


def _scan_plain(s):
    c, T = s["case"], s["x"].dtype
    B, L, D, N, G = c["B"], c.get("L", 1), c["D"], c["N"], c["G"]
    kind = c["kind"]
    step = kind == "scan_step"

    def rows(k):        # [B, L, ...] in 32 bits, also where the call has one token
        return None if s[k] is None else (s[k][:, None] if step else s[k]).float()

    def heads(v):       # [B, L, G, N] -> [B, L, D, N]
        return v.repeat_interleave(D // G, dim=2)

    x, z, raw, Bm, Cm = (rows(k) for k in ("x", "z", "dt", "B", "C"))
    A, skip = s["A"], s["skip"]
    v = raw + s["dt_bias"]
    dt = torch.logaddexp(v, torch.zeros_like(v))
    if s.get("lens") is not None:   # behind a prompt's end: nothing decays, nothing comes in
        inside = (torch.arange(L, device=x.device)[None] < s["lens"][:, None])[:, :, None]
        dt = dt * inside
    a = torch.exp(dt[..., None] * A)
    b = heads(Bm) * (dt * x)[..., None]
    if step:
        h = a * s["h"][:, None] + b
    else:
        h = _recur(a, b)
    Ch = heads(Cm)
    y0 = (Ch * h).sum(-1) + skip * x
    q = None if z is None else torch.sigmoid(z)
    y = y0 if z is None else y0 * z * q
    if step:
        s["h_out"].copy_(h[:, 0])
        return {"y": y[:, 0].to(T), "h": s["h_out"]}
    last = h[:, -1].clone()
    if kind == "scan":
        if s["lens"] is not None:
            y = y * inside
        return {"y": y.to(T), "h": last}
    dy = s["dy"].float()
    dz = None if z is None else dy * y0 * q * (1 + z * (1 - q))
    dy = dy if z is None else dy * z * q
    # the adjoint of the state runs backwards, each token's with the decay of the token after it
    after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], dim=1)
    gh = _recur(after.flip(1), (Ch * dy[..., None]).flip(1)).flip(1)
    before = torch.cat([torch.zeros_like(h[:, :1]), h[:, :-1]], dim=1)
    da = gh * before * a
    in_ = (gh * heads(Bm)).sum(-1)
    ddt = (da * A).sum(-1) + in_ * x
    ddt = ddt * torch.sigmoid(v)
    out = {"y": y.to(T), "h": last, "dx": (in_ * dt + skip * dy).to(T), "ddt": ddt.to(T),
           "dA": (da * dt[..., None]).sum((0, 1)),
           "dB": (gh * (dt * x)[..., None]).view(B, L, G, D // G, N).sum(3).to(T),
           "dC": (h * dy[..., None]).view(B, L, G, D // G, N).sum(3).to(T),
           "dskip": (dy * x).sum((0, 1)), "ddt_bias": ddt.sum((0, 1))}
    if z is not None:
        out["dz"] = dz.to(T)
    return out


# --------------------------------------------------------------------------
# the definitions in 64 bits, token by token and group by group
# --------------------------------------------------------------------------
def exact(case, seed):
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in prepare(case, seed).items()}
    c, kind = s["case"], s["case"]["kind"]
    f = _norm_exact if kind.startswith("norm") else _conv_exact if kind.startswith("conv") else _scan_exact
    with torch.no_grad():
        return {k: np.array(v.cpu().numpy()) for k, v in f(s, c).items()}


def _silu64(u):
    return u / (1 + torch.exp(-u))


def _dsilu64(u):
    p = 1 / (1 + torch.exp(-u))
    return p + u * p * (1 - p)


ACT64 = {"none": lambda u: u, "relu": lambda u: u.clamp(min=0), "silu": _silu64}
SLOPE64 = {"none": lambda u: u * 0 + 1, "relu": lambda u: (u > 0) * 1.0, "silu": _dsilu64}


def _norm_exact(s, c):
    x, w, b, n = s["x"], s["weight"], s["bias"], c["C"] // c["G"]
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.zeros_like(w), torch.zeros_like(w)
    for k in range(0, c["C"], n):
        part, ws, bs = x[:, :, k:k + n], w[k:k + n], b[k:k + n]
        m = part.sum((1, 2), keepdim=True) / (c["S"] * n)
        r = 1 / torch.sqrt(((part - m) ** 2).sum((1, 2), keepdim=True) / (c["S"] * n) + 1e-5)
        unit = (part - m) * r
        u = unit * ws + bs
        y[:, :, k:k + n] = ACT64[c["act"]](u)
        if c["kind"] == "norm_train":
            du = s["dy"][:, :, k:k + n] * SLOPE64[c["act"]](u)
            dw[k:k + n], db[k:k + n] = (du * unit).sum((0, 1)), du.sum((0, 1))
            t = du * ws
            m1, m2 = t.sum((1, 2), keepdim=True) / (c["S"] * n), (t * unit).sum((1, 2), keepdim=True) / (c["S"] * n)
            dx[:, :, k:k + n] = (t - m1 - unit * m2) * r
    return {"y": y, "dx": dx, "dw": dw, "db": db} if c["kind"] == "norm_train" else {"y": y}


def _conv_exact(s, c):
    w, b, K, D, B = s["weight"], s["bias"], c["K"], c["D"], c["B"]
    if c["kind"] == "conv_step":
        u = b + s["x"] * w[:, K - 1]
        for a in range(K - 1):
            u = u + s["kept"][:, a] * w[:, a]
        return {"y": ACT64[c["act"]](u), "kept": torch.cat([s["kept"], s["x"][:, None]], 1)[:, 1:]}
    x, L = s["x"], c["L"]
    u = b + torch.zeros_like(x)
    for a in range(K):
        back = K - 1 - a
        if back < L:
            u[:, back:] += w[:, a] * x[:, :L - back]
    y = ACT64[c["act"]](u)
    if c["kind"] == "conv":
        final = x.new_zeros(B, K - 1, D)
        for i in range(B):
            n = L if s["lens"] is None else int(s["lens"][i])
            y[i, n:] = 0
            m = min(n, K - 1)
            if m:
                final[i, K - 1 - m:] = x[i, n - m:n]
        return {"y": y, "final": final}
    du = s["dy"] * SLOPE64[c["act"]](u)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    for a in range(K):
        back = K - 1 - a
        if back < L:
            dx[:, :L - back] += w[:, a] * du[:, back:]
            dw[:, a] = (du[:, back:] * x[:, :L - back]).sum((0, 1))
    return {"y": y, "dx": dx, "dw": dw, "db": du.sum((0, 1))}


def _scan_exact(s, c):
    B, D, N, G, L = c["B"], c["D"], c["N"], c["G"], c.get("L", 1)
    kind, A, skip = c["kind"], s["A"], s["skip"]
    group = torch.arange(D, device=A.device) // (D // G)
    v = s["dt"] + s["dt_bias"]
    dt = torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))
    if kind == "scan_step":
        h = torch.exp(dt[..., None] * A) * s["h"] + (dt * s["x"])[..., None] * s["B"][:, group]
        return {"y": ((h * s["C"][:, group]).sum(-1) + skip * s["x"]) * _silu64(s["z"]), "h": h}
    x, z, lens = s["x"], s["z"], s.get("lens")
    train = kind == "scan_train"
    h, y0 = A.new_zeros(B, D, N), torch.zeros_like(x)
    kept = A.new_empty(L, B, D, N) if train else None
    for t in range(L):
        new = torch.exp(dt[:, t, :, None] * A) * h + (dt[:, t] * x[:, t])[..., None] * s["B"][:, t, group]
        h = new if lens is None else torch.where((t < lens)[:, None, None], new, h)
        y0[:, t] = (h * s["C"][:, t, group]).sum(-1) + skip * x[:, t]
        if train:
            kept[t] = h
    y = y0 if z is None else y0 * _silu64(z)
    if not train:
        if lens is not None:
            y = y * (torch.arange(L, device=x.device)[None] < lens[:, None])[:, :, None]
        return {"y": y, "h": h}
    dy0 = s["dy"] if z is None else s["dy"] * _silu64(z)
    dx, ddt = torch.empty_like(x), torch.empty_like(x)
    dB, dC, dA = torch.zeros_like(s["B"]), torch.zeros_like(s["C"]), torch.zeros_like(A)
    carry = A.new_zeros(B, D, N)
    for t in range(L - 1, -1, -1):
        lam = carry + dy0[:, t, :, None] * s["C"][:, t, group]
        decay = torch.exp(dt[:, t, :, None] * A)
        into = (lam * s["B"][:, t, group]).sum(-1)
        by_decay = lam * decay * kept[t - 1] if t else torch.zeros_like(lam)
        dx[:, t] = into * dt[:, t] + skip * dy0[:, t]
        ddt[:, t] = into * x[:, t] + (by_decay * A).sum(-1)
        dA += (by_decay * dt[:, t, :, None]).sum(0)
        dB[:, t] = (lam * (dt[:, t] * x[:, t])[..., None]).view(B, G, D // G, N).sum(2)
        dC[:, t] = (kept[t] * dy0[:, t, :, None]).view(B, G, D // G, N).sum(2)
        carry = lam * decay
    ddt = ddt / (1 + torch.exp(-v))
    out = {"y": y, "h": h, "dx": dx, "ddt": ddt, "dA": dA, "dB": dB, "dC": dC, "dskip": (dy0 * x).sum((0, 1)),
           "ddt_bias": ddt.sum((0, 1))}
    if z is not None:
        out["dz"] = s["dy"] * y0 * _dsilu64(z)
    return out
