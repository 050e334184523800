#!/usr/bin/env python3
"""A token mixer from the library's sequence operators, trained and then sampled.

    python examples/token_mixer.py [--steps 150]

One block: a projection gives x and a gate z; a short causal convolution with SiLU over x; from its result a projection
gives the scan's steps, B and C; the selective scan, gated by z; a group norm per token (statistics over the channels of
a head); a projection back.  Matrix products are PyTorch's, everything along the sequence is the library's:

  training    merit_causal_conv, merit_scan, merit_group_norm and their backward passes, as torch.autograd functions
  a prompt    the same forward calls, with the prompt's length for each sequence, leaving the states behind
  sampling    merit_causal_conv_step and merit_scan_step, one token at a time, on those states, in place

The task: a sequence of symbols repeats with a period of its own; predict the next symbol.  Sampling continues a prompt.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1911_03458_amd import binding as mb  # noqa: E402

DEV = "cuda:0"
_plans = {}


def plan(make, *sizes):
    """The plan for these sizes, made once."""
    if (make, sizes) not in _plans:
        _plans[make, sizes] = make(*sizes)
    return _plans[make, sizes]


def conv_plan(B, L, D, K):
    return plan(mb.merit_plan_causal_conv, mb.MERIT_BF16, B, L, D, K, mb.MERIT_ACT_SILU)


def scan_plan(B, L, D, N):
    return plan(mb.merit_plan_scan, mb.MERIT_BF16, B, L, D, N)


def norm_plan(tokens, D, heads):
    return plan(mb.merit_plan_group_norm, mb.MERIT_BF16, tokens, 1, D, heads)


class CausalConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        ctx.save_for_backward(x, weight, bias)
        return mb.merit_causal_conv(conv_plan(*x.shape, weight.shape[1]), x, weight, bias)

    @staticmethod
    def backward(ctx, dy):
        x, weight, bias = ctx.saved_tensors
        return mb.merit_causal_conv_backward(conv_plan(*x.shape, weight.shape[1]), dy.contiguous(), x, weight, bias)


class Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, A, B, C, skip, z, dt_bias):
        y, states = mb.merit_scan(scan_plan(*x.shape, A.shape[1]), x, dt, A, B, C, skip=skip, z=z, dt_bias=dt_bias, states=True)
        ctx.save_for_backward(x, dt, A, B, C, skip, z, dt_bias, states)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, dt, A, B, C, skip, z, dt_bias, states = ctx.saved_tensors
        g = mb.merit_scan_backward(scan_plan(*x.shape, A.shape[1]), dy.contiguous(), x, dt, A, B, C, states, skip=skip, z=z,
                                   dt_bias=dt_bias)
        return tuple(g[k] for k in ("dx", "ddt", "dA", "dB", "dC", "dskip", "dz", "ddt_bias"))


class GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, heads):
        rows = x.reshape(-1, 1, x.shape[-1])
        y, mean, rstd = mb.merit_group_norm(norm_plan(rows.shape[0], x.shape[-1], heads), rows, weight, bias, stats=True)
        ctx.save_for_backward(rows, weight, bias, mean, rstd)
        ctx.heads = heads
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, dy):
        rows, weight, bias, mean, rstd = ctx.saved_tensors
        dx, dw, db = mb.merit_group_norm_backward(norm_plan(rows.shape[0], rows.shape[2], ctx.heads),
                                                  dy.reshape(rows.shape).contiguous(), rows, mean, rstd, weight, bias)
        return dx.view(dy.shape), dw, db, None


class Mixer(torch.nn.Module):
    def __init__(self, symbols, width=64, inner=128, states=16, taps=4, heads=4, rank=8):
        super().__init__()
        self.N, self.K, self.heads, self.rank, self.inner = states, taps, heads, rank, inner
        self.embed = torch.nn.Embedding(symbols, width)
        self.into = torch.nn.Linear(width, 2 * inner, bias=False)
        self.side = torch.nn.Linear(inner, rank + 2 * states, bias=False)
        self.step = torch.nn.Linear(rank, inner, bias=False)
        self.out = torch.nn.Linear(inner, width, bias=False)
        self.head = torch.nn.Linear(width, symbols)
        self.taps = torch.nn.Parameter(torch.randn(inner, taps) / math.sqrt(taps))
        self.taps_bias = torch.nn.Parameter(torch.zeros(inner))
        self.log_A = torch.nn.Parameter(torch.log(torch.arange(1, states + 1).float()).repeat(inner, 1))
        self.skip = torch.nn.Parameter(torch.ones(inner))
        self.dt_bias = torch.nn.Parameter(torch.log(torch.expm1(torch.exp(torch.empty(inner).uniform_(math.log(1e-2), math.log(0.3))))))
        self.norm_w, self.norm_b = torch.nn.Parameter(torch.ones(inner)), torch.nn.Parameter(torch.zeros(inner))

    def _side(self, x):
        """The scan's steps, B and C of some tokens: slices of one projection."""
        rank, b, c = self.side(x).split([self.rank, self.N, self.N], dim=-1)
        return self.step(rank), b.unsqueeze(-2), c.unsqueeze(-2)

    def forward(self, symbols):
        with torch.autocast("cuda", dtype=torch.bfloat16):
            e = self.embed(symbols)
            x, z = self.into(e).split(self.inner, dim=-1)
            x = CausalConv.apply(x, self.taps, self.taps_bias)
            dt, B, C = self._side(x)
            y = Scan.apply(x, dt, -torch.exp(self.log_A), B, C, self.skip, z, self.dt_bias)
            y = GroupNorm.apply(y, self.norm_w, self.norm_b, self.heads)
            return self.head(e + self.out(y))

    @torch.no_grad()
    def prompt(self, symbols, lens):
        """The logits behind each prompt's last symbol, and the states to go on from."""
        B, L = symbols.shape
        with torch.autocast("cuda", dtype=torch.bfloat16):
            e = self.embed(symbols)
            x, z = self.into(e).split(self.inner, dim=-1)
            x, kept = mb.merit_causal_conv(conv_plan(B, L, self.inner, self.K), x, self.taps, self.taps_bias, lens=lens, final=True)
            dt, Bm, C = self._side(x)
            y, h = mb.merit_scan(scan_plan(B, L, self.inner, self.N), x, dt, -torch.exp(self.log_A), Bm, C, skip=self.skip, z=z,
                                 dt_bias=self.dt_bias, lens=lens, final=True)
            last = (lens.long() - 1)[:, None, None]
            y = y.gather(1, last.expand(-1, 1, self.inner))
            y = mb.merit_group_norm(norm_plan(B, self.inner, self.heads), y, self.norm_w, self.norm_b)
            e = e.gather(1, last.expand(-1, 1, e.shape[2]))
            return self.head(e + self.out(y))[:, 0], (kept, h)

    @torch.no_grad()
    def next(self, symbols, state):
        """One symbol more for every sequence, on its states, in place."""
        kept, h = state
        B = symbols.shape[0]
        with torch.autocast("cuda", dtype=torch.bfloat16):
            e = self.embed(symbols)
            x, z = self.into(e).split(self.inner, dim=-1)
            x, _ = mb.merit_causal_conv_step(conv_plan(B, 1, self.inner, self.K), kept, x, self.taps, self.taps_bias, kept_out=kept)
            dt, Bm, C = self._side(x)
            y, _ = mb.merit_scan_step(scan_plan(B, 1, self.inner, self.N), h, x, dt, -torch.exp(self.log_A), Bm, C, skip=self.skip, z=z,
                                      dt_bias=self.dt_bias, h_out=h)
            y = mb.merit_group_norm(norm_plan(B, self.inner, self.heads), y[:, None], self.norm_w, self.norm_b)[:, 0]
            return self.head(e + self.out(y))


def batch(B, L, symbols, g, periods=(2, 3, 4)):
    """Sequences that repeat themselves."""
    out = torch.empty(B, L, dtype=torch.long)
    for b in range(B):
        p = periods[int(torch.randint(len(periods), (1,), generator=g))]
        out[b] = torch.randint(symbols, (p,), generator=g).repeat(L // p + 1)[:L]
    return out.to(DEV)


def train(steps=150, B=32, L=65, symbols=12, seed=0, log=print):
    torch.manual_seed(seed)
    g = torch.Generator().manual_seed(seed)
    model = Mixer(symbols).to(DEV)
    opt = torch.optim.AdamW(model.parameters(), lr=4e-3)
    losses = []
    for i in range(steps):
        seq = batch(B, L, symbols, g)
        logits = model(seq[:, :-1])
        loss = torch.nn.functional.cross_entropy(logits.float().flatten(0, 1), seq[:, 1:].flatten())
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
        if i % 25 == 0 or i == steps - 1:
            log(f"step {i:4d}  loss {losses[-1]:.3f}", flush=True)
    return model, losses, g


def sample(model, seq, lens, new):
    """`new` symbols behind the first lens[b] of each row of seq: the likeliest each time."""
    logits, state = model.prompt(seq, lens)
    got = [logits.argmax(-1)]
    for _ in range(new - 1):
        got.append(model.next(got[-1], state).argmax(-1))
    return torch.stack(got, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=150)
    a = ap.parse_args()
    model, _, g = train(a.steps)
    seq = batch(6, 40, 12, g)
    lens = torch.tensor([24, 20, 17, 24, 13, 9], dtype=torch.int32, device=DEV)
    got = sample(model, seq[:, :24].contiguous(), lens, 10)
    for b, n in enumerate(lens.tolist()):
        want = seq[b, n:n + 10].tolist()
        print("prompt", seq[b, :n].tolist()[-8:], "->", got[b].tolist(), "as it goes on" if got[b].tolist() == want else f"goes on {want}")


if __name__ == "__main__":
    main()
