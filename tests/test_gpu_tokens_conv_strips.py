"""The causal convolution on strips of every length: 8, 16 and 32 tokens forward, 16, 32 and 64 backward (a lane walks down a
strip; short ones are what few tokens get), four channels a lane and one, strips that sequences fill and do not.
Chains as in test_gpu_tokens_conv: 32; a gradient of a parameter 128 + B L / 8."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import token_reference as ref                          # noqa: E402
from oracle import tokens as ot                        # noqa: E402
from token_helpers import ACTS, DEV, TYPES, check, host     # noqa: E402

CHAIN = 32


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


def _strip(B, L, D, backward):
    """The plan's rule (csrc/token_plan.cpp), so that the shapes below are what they say."""
    units, strip = D // 4 if D % 4 == 0 else D, 64 if backward else 32
    while strip > 8 and B * -(-L // strip) * units < (2 if backward else 4) * 65536:
        strip //= 2
    return strip


# B, L, D, K, the strips forward and backward.  Channels: whole wavefronts of units, and not
CASES = [(3, 6000, 512, 4, 8, 16), (3, 6001, 1032, 4, 16, 32), (3, 5603, 2048, 4, 32, 64), (3, 5600, 2052, 3, 32, 64),
         (4, 4416, 1024, 8, 16, 32), (3, 5601, 2048, 2, 32, 64), (1, 16800, 2048, 1, 32, 64), (9, 1900, 1000, 7, 16, 32),
         (3, 6001, 127, 4, 8, 16), (3, 6000, 255, 4, 16, 32), (3, 5709, 513, 4, 32, 64), (2, 8600, 513, 8, 32, 64),
         (3, 5700, 515, 2, 32, 64), (1, 17100, 513, 1, 32, 64), (60, 300, 255, 5, 16, 32), (4, 4300, 257, 6, 16, 32),
         (600, 65, 130, 3, 16, 64), (64, 512, 260, 3, 8, 16)]


def _inputs(B, L, D, K, dtype):
    T = TYPES[dtype][0]
    g = torch.Generator(device=DEV).manual_seed(B + L + D + K)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)

    lens = torch.randint(0, L + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    lens[0] = L
    if B > 1:
        lens[1] = 64 * (L // 128)                       # a sequence that ends where a strip does
    if B > 2:
        lens[2] = 0 if B > 8 else 1
    return dict(x=normal(B, L, D, dtype=T), w=normal(D, K, std=K ** -0.5), b=normal(D, std=0.3), init=normal(B, K - 1, D, dtype=T),
                dy=normal(B, L, D, dtype=T), dfinal=normal(B, K - 1, D, dtype=T), lens=lens)


@pytest.mark.parametrize("B, L, D, K, forward, backward", CASES)
def test_strips(mb, B, L, D, K, forward, backward):
    assert (_strip(B, L, D, False), _strip(B, L, D, True)) == (forward, backward)
    dtype = ("bf16", "f32", "f16")[(B + L + D) % 3]
    v = _inputs(B, L, D, K, dtype)
    many = 128 + B * L // 8
    for kind, b, init, lens, dfinal in (("silu", v["b"], None, None, None), ("silu", v["b"], v["init"], v["lens"], v["dfinal"]),
                                        ("none", None, v["init"], v["lens"], None)):
        plan = mb.merit_plan_causal_conv(TYPES[dtype][1], B, L, D, K, ACTS[kind])
        y, final = mb.merit_causal_conv(plan, v["x"], v["w"], b, init=init, lens=lens, final=True)
        want = ref.causal_conv(v["x"], v["w"], b, init, lens, kind)
        ref.near(y, want[0], CHAIN, "y")
        assert torch.equal(final.double(), want[1])
        got = mb.merit_causal_conv_backward(plan, v["dy"], v["x"], v["w"], b, init=init, lens=lens, dfinal=dfinal, dinit=True)
        want = ref.causal_conv_backward(v["dy"], v["x"], v["w"], b, init, lens, dfinal, kind)
        for t, r, what, chain in zip(got, want, ("dx", "dw", "db", "dinit"), (2 * CHAIN, many, many, 2 * CHAIN)):
            if r.numel():
                ref.near(t, r, chain, what)


def test_nothing_behind_an_end_is_read(mb):
    """Whole strips beside strips that end early: NaN behind each sequence's end, in x and dy."""
    B, L, D, K = 3, 5700, 513, 4
    v = _inputs(B, L, D, K, "f16")
    plan = mb.merit_plan_causal_conv(TYPES["f16"][1], B, L, D, K, ACTS["silu"])
    kw = dict(init=v["init"], lens=v["lens"])
    y = mb.merit_causal_conv(plan, v["x"], v["w"], v["b"], **kw)
    grads = mb.merit_causal_conv_backward(plan, v["dy"], v["x"], v["w"], v["b"], **kw)
    behind = torch.arange(L, device=DEV)[None] >= v["lens"][:, None]
    x, dy = v["x"].masked_fill(behind[..., None], float("nan")), v["dy"].masked_fill(behind[..., None], float("nan"))
    assert torch.equal(mb.merit_causal_conv(plan, x, v["w"], v["b"], **kw), y)
    for a, b in zip(mb.merit_causal_conv_backward(plan, dy, x, v["w"], v["b"], **kw), grads):
        assert torch.equal(a, b)


def test_the_reference(mb):
    """token_reference against the oracle."""
    v = _inputs(5, 19, 6, 4, "f32")
    v["lens"][3] = 2
    h = {k: host(t) for k, t in v.items()}
    lens = v["lens"].cpu().numpy()
    for kind, init, n, dfinal in (("silu", "init", lens, "dfinal"), ("none", None, None, None), ("relu", "init", lens, None)):
        args = dict(bias=v["b"], init=v["init"] if init else None, lens=None if n is None else v["lens"], kind=kind)
        oargs = dict(bias=h["b"], init=h["init"] if init else None, lens=n, kind=kind)
        pairs = list(zip(ref.causal_conv(v["x"], v["w"], **args), ot.causal_conv(h["x"], h["w"], **oargs)))
        pairs += zip(ref.causal_conv_backward(v["dy"], v["x"], v["w"], dfinal=v["dfinal"] if dfinal else None, **args),
                     ot.causal_conv_backward(h["dy"], h["x"], h["w"], dfinal=h["dfinal"] if dfinal else None, **oargs))
        for a, b in pairs:
            np.testing.assert_allclose(a.cpu().numpy(), b, rtol=1e-12, atol=1e-12)
