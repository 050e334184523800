"""Inputs and comparisons of the token operators' tests.

Tolerances.  A result of type T is fp32 arithmetic rounded once: half an ulp of T, 2^-24, 2^-11 or 2^-8 of it (`UNIT`).
The fp32 arithmetic before it: a chain of at most `chain` roundings, each at most 2^-24 of the largest value in the chain,
which for these inputs (values around one, decays below one) is taken as 16 times the results' root mean square or the
result itself, whichever is larger.  `chain` is the length of the longest chain of the operator at that size: the terms
of a sum, the tokens of a recurrence times the four roundings of a token, twice that for a gradient through it."""
import numpy as np
import torch

from paper_1911_03458_amd import binding as mb

DEV = "cuda:0"
TYPES = {"f32": (torch.float32, mb.MERIT_F32, 2.0 ** -24), "f16": (torch.float16, mb.MERIT_F16, 2.0 ** -11),
         "bf16": (torch.bfloat16, mb.MERIT_BF16, 2.0 ** -8)}
ACTS = {"none": mb.MERIT_ACT_NONE, "relu": mb.MERIT_ACT_RELU, "silu": mb.MERIT_ACT_SILU}


class Gen:
    """Seeded values on the CPU, rounded to a type, as device tensors."""

    def __init__(self, seed):
        self.rng = np.random.default_rng(seed)

    def normal(self, *shape, dtype=torch.float32, mean=0.0, std=1.0):
        return torch.from_numpy(self.rng.normal(mean, std, size=shape)).to(dtype).to(DEV)

    def uniform(self, *shape, dtype=torch.float32, lo=0.0, hi=1.0):
        return torch.from_numpy(self.rng.uniform(lo, hi, size=shape)).to(dtype).to(DEV)


def wider(t, front=3, back=5, value=float("nan")):
    """The same values as a slice of rows `front` + `back` channels wider, the rest of which is `value`."""
    big = torch.full(t.shape[:-1] + (t.shape[-1] + front + back,), value, dtype=t.dtype, device=t.device)
    big[..., front:front + t.shape[-1]] = t
    return big[..., front:front + t.shape[-1]]


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def check(got, want, chain, what):
    """got: a device tensor; want: the 64-bit result."""
    unit = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[got.dtype]
    assert tuple(got.shape) == want.shape, (what, tuple(got.shape), want.shape)
    g = host(got)
    assert np.isfinite(g).all() == np.isfinite(want).all(), what
    if not want.size:
        return
    rms = np.sqrt(np.mean(want ** 2))
    # (below a type's normal range its steps are 2^-24 of binary16 and next to nothing of the others)
    tiny = 2.0 ** -24 if got.dtype == torch.float16 else 2.0 ** -126
    bound = 1.01 * unit * np.abs(want) + tiny + chain * 2.0 ** -24 * np.maximum(16 * rms, np.abs(want))
    err = np.abs(g - want)
    assert (err <= bound).all(), (what, float((err / bound).max()), float(err.max()), np.unravel_index(np.argmax(err / bound), err.shape))
