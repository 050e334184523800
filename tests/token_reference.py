"""The token operators' definitions in 64 bits on the device, whole tensors at a time, for sizes that oracle/tokens.py would walk
for too long (test_gpu_tokens_conv_strips and test_gpu_tokens_norm_forms pin them against it at small ones), and the comparison of
token_helpers on the device."""
import torch


def near(got, want, chain, what):
    """token_helpers.check, with `want` on the device."""
    unit = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[got.dtype]
    assert got.shape == want.shape, (what, got.shape, want.shape)
    g = got.double()
    assert bool(torch.isfinite(want).all()) and bool(torch.isfinite(g).all()), what
    rms = want.square().mean().sqrt()
    tiny = 2.0 ** -24 if got.dtype == torch.float16 else 2.0 ** -126
    bound = 1.01 * unit * want.abs() + tiny + chain * 2.0 ** -24 * torch.maximum(16 * rms, want.abs())
    ratio = (g - want).abs() / bound
    assert float(ratio.max()) <= 1.0, (what, float(ratio.max()), int(ratio.argmax()), tuple(got.shape))


def act(u, kind):
    return u / (1.0 + torch.exp(-u)) if kind == "silu" else u.clamp(min=0) if kind == "relu" else u


def act_slope(u, kind):
    if kind == "silu":
        q = 1.0 / (1.0 + torch.exp(-u))
        return q * (1.0 + u * (1.0 - q))
    return (u > 0).double() if kind == "relu" else torch.ones_like(u)


def _inside(x, lens):
    B, L, _ = x.shape
    n = torch.full((B,), L, device=x.device) if lens is None else lens.long().clamp(0, L)
    return n, (torch.arange(L, device=x.device)[None] < n[:, None])[:, :, None]


def _rows(x, init, K, n, inside):
    """[B, K - 1 + L, D]: (init, x), zeros behind a sequence's end, and where its last K - 1 rows are"""
    B, L, D = x.shape
    first = x.new_zeros(B, K - 1, D) if init is None else init.double()
    last = (n[:, None] + torch.arange(K - 1, device=x.device))[:, :, None].expand(-1, -1, D)
    return torch.cat([first, torch.where(inside, x.double(), 0.0)], 1), last


def _before(rows, w, b, K, L):
    u = sum(w[:, a] * rows[:, a:a + L] for a in range(K))
    return u if b is None else u + b


def causal_conv(x, weight, bias=None, init=None, lens=None, kind="none"):
    (_, L, _), K = x.shape, weight.shape[1]
    n, inside = _inside(x, lens)
    rows, last = _rows(x, init, K, n, inside)
    u = _before(rows, weight.double(), None if bias is None else bias.double(), K, L)
    return torch.where(inside, act(u, kind), 0.0), rows.gather(1, last)


def causal_conv_backward(dy, x, weight, bias=None, init=None, lens=None, dfinal=None, kind="none"):
    (_, L, _), K = x.shape, weight.shape[1]
    n, inside = _inside(x, lens)
    w = weight.double()
    rows, last = _rows(x, init, K, n, inside)
    u = _before(rows, w, None if bias is None else bias.double(), K, L)
    du = torch.where(inside, dy.double() * act_slope(u, kind), 0.0)
    drows, dw = torch.zeros_like(rows), torch.empty_like(w)
    for a in range(K):
        drows[:, a:a + L] += w[:, a] * du
        dw[:, a] = (du * rows[:, a:a + L]).sum((0, 1))
    if dfinal is not None:
        drows.scatter_add_(1, last, dfinal.double())
    return torch.where(inside, drows[:, K - 1:], 0.0), dw, du.sum((0, 1)), drows[:, :K - 1]


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, kind="none"):
    N, S, C = x.shape
    v = x.double().view(N, S, groups, C // groups)
    mean = v.mean((1, 3), keepdim=True)
    rstd = 1.0 / torch.sqrt((v - mean).square().mean((1, 3), keepdim=True) + eps)
    u = ((v - mean) * rstd).view(N, S, C)
    u = u if weight is None else u * weight.double()
    u = u if bias is None else u + bias.double()
    return act(u, kind), mean.view(N, groups), rstd.view(N, groups)


def group_norm_backward(dy, x, groups, weight=None, bias=None, eps=1e-5, kind="none"):
    N, S, C = x.shape
    _, mean, rstd = group_norm(x, groups, eps=eps)
    rstd = rstd.view(N, 1, groups, 1)
    xh = (x.double().view(N, S, groups, -1) - mean.view(N, 1, groups, 1)) * rstd
    w = torch.ones(C, device=x.device, dtype=torch.float64) if weight is None else weight.double()
    u = xh.reshape(N, S, C) * w
    du = dy.double() * act_slope(u if bias is None else u + bias.double(), kind)
    g = (du * w).view(N, S, groups, -1)
    dx = rstd * (g - g.mean((1, 3), keepdim=True) - xh * (g * xh).mean((1, 3), keepdim=True))
    return dx.view(N, S, C), (du * xh.view(N, S, C)).sum((0, 1)), du.sum((0, 1))
