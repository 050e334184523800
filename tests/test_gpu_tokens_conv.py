"""Short causal convolution against the 64-bit definition: forward, backward, single tokens (tolerances: token_helpers).
Chain: K products and the bias, the activation: 32; a gradient of a parameter sums B L terms in pieces: 128 + B L / 8."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import tokens as ot                        # noqa: E402
from token_helpers import ACTS, DEV, TYPES, Gen, check, host, wider     # noqa: E402

CHAIN = 32


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


SHAPES = [(1, 1, 8, 4), (2, 3, 64, 4), (1, 2, 5, 4), (3, 33, 40, 4), (2, 65, 136, 3), (1, 200, 8, 2), (2, 17, 7, 1), (1, 50, 520, 4),
          (2, 40, 24, 5), (1, 19, 16, 6), (2, 9, 33, 7), (2, 70, 16, 8), (40, 2, 16, 4), (1, 130, 1, 4)]


def _inputs(shape, dtype, seed):
    B, L, D, K = shape
    T = TYPES[dtype][0]
    g = Gen(seed)
    return dict(x=g.normal(B, L, D, dtype=T), w=g.normal(D, K, std=K ** -0.5), b=g.normal(D, std=0.3),
                init=g.normal(B, K - 1, D, dtype=T), dy=g.normal(B, L, D, dtype=T), dfinal=g.normal(B, K - 1, D, dtype=T),
                lens=torch.from_numpy(g.rng.integers(-1, L + 2, size=B).astype(np.int32)).to(DEV))


def _plan(mb, shape, dtype, act):
    return mb.merit_plan_causal_conv(TYPES[dtype][1], *shape, ACTS[act])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(mb, shape, dtype):
    v = _inputs(shape, dtype, sum(shape))
    for act, b, init, lens in (("silu", v["b"], None, None), ("none", None, v["init"], None), ("relu", v["b"], v["init"], v["lens"]),
                               ("none", v["b"], None, v["lens"])):
        y, final = mb.merit_causal_conv(_plan(mb, shape, dtype, act), v["x"], v["w"], b, init=init, lens=lens, final=True)
        want = ot.causal_conv(host(v["x"]), host(v["w"]), host(b), host(init), None if lens is None else lens.cpu(), act)
        check(y, want[0], CHAIN, "y")
        assert np.array_equal(host(final), want[1])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(mb, shape, dtype):
    v = _inputs(shape, dtype, sum(shape) + 1)
    many = 128 + shape[0] * shape[1] // 8
    for act, b, init, lens, dfinal in (("silu", v["b"], None, None, None), ("none", None, v["init"], None, v["dfinal"]),
                                       ("silu", v["b"], v["init"], v["lens"], v["dfinal"])):
        got = mb.merit_causal_conv_backward(_plan(mb, shape, dtype, act), v["dy"], v["x"], v["w"], b, init=init, lens=lens,
                                            dfinal=dfinal, dinit=True)
        want = ot.causal_conv_backward(host(v["dy"]), host(v["x"]), host(v["w"]), host(b), host(init),
                                       None if lens is None else lens.cpu(), host(dfinal), act)
        for g, r, what, chain in zip(got, want, ("dx", "dw", "db", "dinit"), (2 * CHAIN, many, many, 2 * CHAIN)):
            check(g, r, chain, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_sequence_in_parts(mb, dtype):
    """A prompt, its rest, then single tokens: the same values as at once, bit for bit, in place and not."""
    B, L, D, K = 3, 21, 40, 4
    v = _inputs((B, L, D, K), dtype, 2)
    y, final = mb.merit_causal_conv(_plan(mb, (B, L, D, K), dtype, "silu"), v["x"], v["w"], v["b"], init=v["init"], final=True)
    kept = v["init"].clone()
    first = mb.merit_causal_conv(_plan(mb, (B, 2, D, K), dtype, "silu"), v["x"][:, :2], v["w"], v["b"], init=kept, final=kept)
    assert first[1] is kept
    parts = [first[0]]
    y2, kept = mb.merit_causal_conv(_plan(mb, (B, 15, D, K), dtype, "silu"), v["x"][:, 2:17], v["w"], v["b"], init=kept, final=True)
    parts.append(y2)
    plan = _plan(mb, (B, 1, D, K), dtype, "silu")
    for t in range(17, L):
        if t % 2:
            yt, kept = mb.merit_causal_conv_step(plan, kept, v["x"][:, t], v["w"], v["b"])
        else:
            yt, same = mb.merit_causal_conv_step(plan, kept, v["x"][:, t], v["w"], v["b"], kept_out=kept)
            assert same is kept
        parts.append(yt[:, None])
    assert torch.equal(torch.cat(parts, 1), y) and torch.equal(kept, final)


@pytest.mark.parametrize("K", [1, 2, 3, 5, 8])
def test_single_tokens(mb, K):
    for dtype, D in (("f16", 24), ("f32", 7), ("bf16", 9)):
        g = Gen(K)
        T = TYPES[dtype][0]
        kept, x, w, b = g.normal(5, K - 1, D, dtype=T), g.normal(5, D, dtype=T), g.normal(D, K), g.normal(D)
        y, out = mb.merit_causal_conv_step(_plan(mb, (5, 1, D, K), dtype, "silu"), kept, x, w, b)
        want, final = ot.causal_conv(host(x)[:, None], host(w), host(b), host(kept), None, "silu")
        check(y, want[:, 0], CHAIN, "y")
        assert np.array_equal(host(out), final)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_slices_and_broadcasts(mb, dtype):
    shape = (3, 20, 24, 4)
    v = _inputs(shape, dtype, 4)
    plan = _plan(mb, shape, dtype, "silu")
    want, final = ot.causal_conv(host(v["x"]), host(v["w"]), host(v["b"]), host(v["init"]), None, "silu")
    grads = ot.causal_conv_backward(host(v["dy"]), host(v["x"]), host(v["w"]), host(v["b"]), host(v["init"]), None, None, "silu")
    for front, back in ((3, 5), (8, 8)):
        out = wider(torch.zeros_like(v["x"]), back, front, 7.0)
        y, f = mb.merit_causal_conv(plan, wider(v["x"], front, back), v["w"].to(v["x"].dtype).float(), v["b"],
                                    init=wider(v["init"], front, back), final=True, y=out)
        assert y is out
        ref = ot.causal_conv(host(v["x"]), host(v["w"].to(v["x"].dtype)), host(v["b"]), host(v["init"]), None, "silu")[0]
        check(y, ref, CHAIN, "y")
        assert np.array_equal(host(f), final) and (out._base[..., :back] == 7.0).all()
        got = mb.merit_causal_conv_backward(plan, wider(v["dy"], front, back), wider(v["x"], back, front), v["w"], v["b"],
                                            init=wider(v["init"], back, front), dinit=True)
        for g, r, what in zip(got, grads, ("dx", "dw", "db", "dinit")):
            check(g, r, 256, what)
    one = v["x"][:1].expand(3, -1, -1)
    same = mb.merit_causal_conv(plan, one, v["w"], v["b"])
    assert torch.equal(same[0], same[2])
    bytime = v["x"].transpose(0, 1).contiguous().transpose(0, 1)      # [L][B][D] in memory
    assert torch.equal(mb.merit_causal_conv(plan, bytime, v["w"], v["b"]), mb.merit_causal_conv(plan, v["x"], v["w"], v["b"]))


def test_what_lies_behind_an_end_is_not_read(mb):
    shape = (4, 40, 16, 4)
    v = _inputs(shape, "f32", 5)
    lens = torch.tensor([0, 1, 17, 40], dtype=torch.int32, device=DEV)
    plan = _plan(mb, shape, "f32", "silu")
    x, dy = v["x"].clone(), v["dy"].clone()
    for b, n in enumerate((0, 1, 17, 40)):
        x[b, n:] = float("nan")
        dy[b, n:] = float("inf")
    for clean, dirty in zip(mb.merit_causal_conv(plan, v["x"], v["w"], v["b"], init=v["init"], lens=lens, final=True),
                            mb.merit_causal_conv(plan, x, v["w"], v["b"], init=v["init"], lens=lens, final=True)):
        assert torch.equal(clean, dirty)
    for clean, dirty in zip(
            mb.merit_causal_conv_backward(plan, v["dy"], v["x"], v["w"], v["b"], init=v["init"], lens=lens, dinit=True),
            mb.merit_causal_conv_backward(plan, dy, x, v["w"], v["b"], init=v["init"], lens=lens, dinit=True)):
        assert torch.equal(clean, dirty)
    # an infinite token reaches itself and the K - 1 after it, in its own channel
    x = v["x"].clone()
    x[2, 20, 5] = float("inf")
    y, clean = (mb.merit_causal_conv(_plan(mb, shape, "f32", "none"), t, v["w"]) for t in (x, v["x"]))
    assert not torch.isfinite(y[2, 20:24, 5]).any()
    y[2, 20:24, 5] = clean[2, 20:24, 5]
    assert torch.equal(y, clean)


def test_nothing_to_do(mb):
    w = torch.ones(16, 4, device=DEV)
    for B, L in ((0, 5), (2, 0)):
        plan = _plan(mb, (B, L, 16, 4), "f32", "silu")
        x, init = torch.empty(B, L, 16, device=DEV), torch.ones(B, 3, 16, device=DEV)
        y, final = mb.merit_causal_conv(plan, x, w, init=init, final=True)
        assert y.shape == x.shape and torch.equal(final, init)
        dx, dw, db, dinit = mb.merit_causal_conv_backward(plan, x, x, w, init=init, dfinal=init, dinit=True)
        assert dx.shape == x.shape and (dw == 0).all() and (db == 0).all() and torch.equal(dinit, init)


def test_offsets_past_32_bits(mb):
    """Rows 2^27 elements apart: the last of 40 begins 10 GB behind the first."""
    B, L, D, K = 1, 40, 64, 4
    big = torch.empty((L - 1) * (1 << 27) + D, dtype=torch.float16, device=DEV)
    x = big.as_strided((B, L, D), (0, 1 << 27, 1))
    v = _inputs((B, L, D, K), "f16", 6)
    x.copy_(v["x"])
    plan = _plan(mb, (B, L, D, K), "f16", "silu")
    y = mb.merit_causal_conv(plan, x, v["w"], v["b"])
    assert torch.equal(y, mb.merit_causal_conv(plan, v["x"], v["w"], v["b"]))
    mb.merit_causal_conv(plan, v["x"], v["w"], v["b"], y=x)
    assert torch.equal(x, y)


def test_refusals(mb):
    plan = _plan(mb, (2, 3, 16, 4), "f16", "none")
    x, w = torch.zeros(2, 3, 16, dtype=torch.float16, device=DEV), torch.zeros(16, 4, device=DEV)
    with pytest.raises(TypeError, match="x: expected"):
        mb.merit_causal_conv(plan, x.float(), w)
    with pytest.raises(ValueError, match="weight: expected shape"):
        mb.merit_causal_conv(plan, x, w.t().contiguous())
    with pytest.raises(TypeError, match="weight"):
        mb.merit_causal_conv(plan, x, None)
    with pytest.raises(TypeError, match="lens"):
        mb.merit_causal_conv(plan, x, w, lens=torch.ones(2, dtype=torch.int64, device=DEV))
    with pytest.raises(TypeError, match="init: expected a device"):
        mb.merit_causal_conv(plan, x, w, init=torch.zeros(2, 3, 16, dtype=torch.float16))
    with pytest.raises(ValueError, match="dense"):
        mb.merit_causal_conv(plan, torch.zeros(2, 3, 32, dtype=torch.float16, device=DEV)[:, :, ::2], w)
    with pytest.raises(ValueError, match="final"):
        mb.merit_causal_conv(plan, x, w, final=x[:, :2])
