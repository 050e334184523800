"""Inputs and the comparison of the tests of the gated delta rule and of the block's norms.

Tolerances.  A result of type T is rounded once, by at most half a step: UNIT of token_helpers, relative to the value.  What comes
before is fp32: a result is reached through products one after the other, each a sum of up to n terms with roundings of 2^-24
of either sign, which grow as the square root of n.  `roundings` is that number: for the delta rule's forward pass four
products of up to 128 terms (K S, the triangular one, K^T u, Q S), 4 sqrt(128) = 45; for gradients those of the other
direction on top, 90; for dg, a sum over a chunk of 64 differences of such products, which cancel, sqrt(64) times as many, 720;
for a row's norms and the sums over rows 4 sqrt(terms of a thread or a tree): at most 64.  Held against the root mean square
of the result (and 8 times that for a single value, where one in a million exceeds five).

y of the 16-bit types is allowed besides what P and u would lose if they went into their product as two bfloat16 terms (the kernels
keep three, and test_gpu_delta_digits holds sums that cancel to DELTA): the second term, at most
2^-8 of the value, is rounded by at most 2^-8 of itself, so 2^-16 of the value is lost at most and, for mantissas and remainders
spread evenly, 2^-17 / sqrt(3) on average (root mean square); the product of two second terms, left out, is as much again.  These
are relative to each term of a sum, so a sum of terms of either sign has as much of its own root mean square: together
sqrt(3) 2^-17 / sqrt(3) = 128 x 2^-24 (`y_of`)."""
import numpy as np

from token_helpers import host

DELTA, GRAD, DECAY, NORM = 45, 90, 720, 64


def y_of(dtype):
    return DELTA if dtype in ("f32", "torch.float32") else DELTA + 128


UNITS = {"torch.float32": 2.0 ** -24, "torch.float16": 2.0 ** -11, "torch.bfloat16": 2.0 ** -8}


def near(got, want, roundings, what, floor=0.0):
    """floor: what values that cancel in `want` are sums of."""
    want = np.asarray(want)
    assert tuple(got.shape) == want.shape, (what, tuple(got.shape), want.shape)
    g, unit = host(got), UNITS[str(got.dtype)]
    if not want.size:
        return
    assert np.isfinite(g).all(), what
    size = max(float(np.sqrt(np.mean(want ** 2))), floor)
    tiny = 2.0 ** -24 if unit == 2.0 ** -11 else 2.0 ** -126
    err = np.abs(g - want)
    bound = 1.01 * unit * np.abs(want) + 8 * roundings * 2.0 ** -24 * np.maximum(size, np.abs(want)) + tiny
    assert (err <= bound).all(), (what, float((err / bound).max()), np.unravel_index(np.argmax(err / bound), err.shape))
    whole = float(np.sqrt(np.mean(err ** 2)))
    assert whole <= 1.01 * unit * size + roundings * 2.0 ** -24 * size + tiny, (what, whole, size)
