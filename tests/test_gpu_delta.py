"""The gated delta rule against the 64-bit definition, forward, backward, one token (tolerances: mixer_helpers)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from mixer_helpers import DECAY, DELTA, GRAD, near, y_of    # noqa: E402
from oracle import mixers as om                         # noqa: E402
from token_helpers import DEV, TYPES, Gen, host, wider  # noqa: E402


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


# B, L, heads, key heads, Dk, Dv: one token, less than a chunk, a chunk and one more, several; keys of one value to the widest, off
# every multiple; value columns off the tiles; shared key heads
SHAPES = [(1, 1, 1, 1, 1, 1), (2, 5, 2, 1, 8, 16), (1, 64, 1, 1, 32, 32), (2, 65, 4, 2, 64, 40), (1, 63, 3, 3, 17, 5),
          (2, 130, 2, 2, 128, 128), (1, 200, 6, 2, 100, 50), (3, 31, 4, 4, 33, 130), (1, 128, 1, 1, 127, 129), (2, 193, 2, 1, 96, 17)]


def _inputs(shape, dtype, seed, unit=True, beta_type=torch.float32):
    B, L, H, K, Dk, Dv = shape
    T, g = TYPES[dtype][0], Gen(seed)
    std = 1.0 if unit else 0.7 * Dk ** -0.5        # (keys of less than unit length: the recurrence does not grow)
    q, k, v = g.normal(B, L, K, Dk, dtype=T, std=std), g.normal(B, L, K, Dk, dtype=T, std=std), g.normal(B, L, H, Dv, dtype=T)
    a = -torch.exp(g.uniform(B, L, H, lo=-6.0, hi=1.0))
    beta = g.uniform(B, L, H, lo=0.05, hi=0.95).to(beta_type)
    return dict(q=q, k=k, v=v, g=a, beta=beta), g


def _h(d):
    return {k: host(t) if isinstance(t, torch.Tensor) else t for k, t in d.items()}


def _plan(mb, shape, dtype, unit=True, **kw):
    B, L, H, K, Dk, Dv = shape
    return mb.merit_plan_delta_rule(TYPES[dtype][1], B, L, H, K, Dk, Dv, normalize=unit, **kw)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(mb, shape, dtype):
    unit = sum(shape) % 2 == 0
    a, g = _inputs(shape, dtype, sum(shape), unit)
    B, L, H, K, Dk, Dv = shape
    h0 = g.normal(B, H, Dk, Dv) if L % 2 else None
    y, h = mb.merit_delta_rule(_plan(mb, shape, dtype, unit), *a.values(), h0=h0, final=True)
    wy, wh, _ = om.delta_rule(**_h(a), h0=host(h0) if h0 is not None else None, scale=Dk ** -0.5, unit=unit)
    near(y, wy, y_of(str(y.dtype)), "y")
    near(h, wh, DELTA, "state")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(mb, shape, dtype):
    unit = sum(shape) % 2 == 1 and shape[4] > 1
    a, g = _inputs(shape, dtype, sum(shape) + 1, unit)
    B, L, H, K, Dk, Dv = shape
    h0, dh = (g.normal(B, H, Dk, Dv), g.normal(B, H, Dk, Dv)) if L % 2 else (None, None)
    dy = g.normal(B, L, H, Dv, dtype=TYPES[dtype][0])
    plan = _plan(mb, shape, dtype, unit)
    _, states = mb.merit_delta_rule(plan, *a.values(), h0=h0, states=True)
    got = mb.merit_delta_rule_backward(plan, dy, a["q"], a["k"], a["g"], a["beta"], states, dh_last=dh, dh0=True)
    want = om.delta_rule_backward(host(dy), **_h(a), h0=None if h0 is None else host(h0), dh_last=None if dh is None else host(dh),
                                  scale=Dk ** -0.5, unit=unit)
    for k, w in want.items():
        # (the last token's decay may have no gradient but what cancels: the products are of its other gradients' size)
        near(got[k], w, DECAY if k == "dg" else GRAD, k, floor=float(np.sqrt(np.mean(want["dbeta"] ** 2))) if k == "dg" else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(2, 100, 1, 1, 29, 10), (1, 228, 1, 1, 31, 40), (2, 100, 2, 1, 100, 24), (1, 165, 2, 2, 33, 16),
                                   (1, 165, 2, 1, 128, 70), (1, 130, 1, 1, 64, 200), (70, 66, 4, 4, 40, 48), (1, 100, 1, 1, 8, 8)])
def test_columns_for_some_of_a_workgroup(mb, shape, dtype):
    """Whole chunks and part of one, with fewer columns than a workgroup has wavefronts for: those without any move rows for the
    others.  With the states kept, without, and backward."""
    a, g = _inputs(shape, dtype, sum(shape) + 2)
    B, L, H, K, Dk, Dv = shape
    plan, dy = _plan(mb, shape, dtype), g.normal(B, L, H, Dv, dtype=TYPES[dtype][0])
    wy, wh, _ = om.delta_rule(**_h(a), scale=Dk ** -0.5)
    y, h = mb.merit_delta_rule(plan, *a.values(), final=True)
    y2, h2, states = mb.merit_delta_rule(plan, *a.values(), final=True, states=True)
    for got in (y, y2):
        near(got, wy, y_of(str(y.dtype)), "y")
    for got in (h, h2):
        near(got, wh, DELTA, "state")
    got = mb.merit_delta_rule_backward(plan, dy, a["q"], a["k"], a["g"], a["beta"], states)
    want = om.delta_rule_backward(host(dy), **_h(a), scale=Dk ** -0.5)
    for k in ("dq", "dk", "dv", "dg", "dbeta"):
        near(got[k], want[k], DECAY if k == "dg" else GRAD, k, floor=float(np.sqrt(np.mean(want["dbeta"] ** 2))) if k == "dg" else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B, H, K, Dk, Dv", [(1, 1, 1, 1, 1), (2, 4, 2, 64, 64), (3, 2, 2, 128, 128), (5, 6, 2, 100, 50), (1, 3, 3, 17, 260), (2, 2, 1, 128, 33)])
def test_one_token(mb, B, H, K, Dk, Dv, dtype):
    unit = Dk % 2 == 0
    a, g = _inputs((B, 1, H, K, Dk, Dv), dtype, Dk + Dv, unit)
    h = g.normal(B, H, Dk, Dv)
    plan = _plan(mb, (B, 1, H, K, Dk, Dv), dtype, unit)
    one = [t[:, 0] for t in a.values()]
    wy, wh, _ = om.delta_rule(**_h(a), h0=host(h), scale=Dk ** -0.5, unit=unit)
    y, out = mb.merit_delta_rule_step(plan, h, *one)
    near(y, wy[:, 0], DELTA, "y")
    near(out, wh, DELTA, "state")
    y2, same = mb.merit_delta_rule_step(plan, h, *one, h_out=h)
    assert same is h and torch.equal(y2, y) and torch.equal(h, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths(mb, dtype):
    """Sequences of no token, one, some, all and more than there are; nothing is read behind them (NaN), results are zeros."""
    shape = (6, 140, 2, 1, 24, 20)
    lens = [0, 1, 64, 100, 140, 1000]
    a, g = _inputs(shape, dtype, 9)
    dy = g.normal(6, 140, 2, 20, dtype=TYPES[dtype][0])
    h0, dh = g.normal(6, 2, 24, 20), g.normal(6, 2, 24, 20)
    for t in (a["q"], a["k"], a["v"], a["g"], a["beta"], dy):
        for b, n in enumerate(lens):
            t[b, n:] = float("nan")
    plan, n = _plan(mb, shape, dtype), torch.tensor(lens, dtype=torch.int32, device=DEV)
    y, h, states = mb.merit_delta_rule(plan, *a.values(), h0=h0, lens=n, final=True, states=True)
    zeros = {k: np.nan_to_num(v) for k, v in _h(a).items()}
    wy, wh, _ = om.delta_rule(**zeros, h0=host(h0), lens=lens, scale=24 ** -0.5)
    near(y, wy, y_of(str(y.dtype)), "y")
    near(h, wh, DELTA, "state")
    got = mb.merit_delta_rule_backward(plan, dy, a["q"], a["k"], a["g"], a["beta"], states, lens=n, dh_last=dh, dh0=True)
    want = om.delta_rule_backward(np.nan_to_num(host(dy)), **zeros, h0=host(h0), lens=lens, dh_last=host(dh), scale=24 ** -0.5)
    for k, w in want.items():
        near(got[k], w, DECAY if k == "dg" else GRAD, k)
    for b, m in enumerate(lens):
        for k in ("dq", "dk", "dv", "dg", "dbeta"):
            assert not got[k][b, m:].any(), k
        assert not y[b, m:].any()
    assert torch.equal(h[0], h0[0]) and torch.equal(got["dh0"][0], dh[0])


@pytest.mark.parametrize("shape", [(2, 70, 4, 2, 40, 24), (2, 70, 2, 2, 64, 64)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views(mb, shape, dtype):
    """Slices of wider rows off every alignment, rows between other rows, a sequence read by all: the same bits as dense ones."""
    a, g = _inputs(shape, dtype, 21, beta_type=TYPES[dtype][0])
    B, L, H, K, Dk, Dv = shape
    plan = _plan(mb, shape, dtype)
    dy = g.normal(B, L, H, Dv, dtype=TYPES[dtype][0])

    def all_of(a, dy):
        y, h, st = mb.merit_delta_rule(plan, *a.values(), final=True, states=True)
        d = mb.merit_delta_rule_backward(plan, dy, a["q"], a["k"], a["g"], a["beta"], st)
        return [y, h] + [d[k] for k in ("dq", "dk", "dv", "dg", "dbeta")]

    def slices(t, front):
        return wider(t.flatten(2), front).unflatten(2, t.shape[2:])

    want = all_of(a, dy)
    for front in (3, 8):
        odd = {k: slices(t, front) for k, t in a.items()}
        assert not odd["q"].is_contiguous()
        assert all(torch.equal(s, t) for s, t in zip(all_of(odd, slices(dy, front)), want))
    strided = {k: torch.stack([t, torch.full_like(t, float("nan"))], 2).flatten(1, 2)[:, ::2] for k, t in a.items()}
    assert all(torch.equal(s, t) for s, t in zip(all_of(strided, dy), want))
    shared = {k: t[:1].expand(t.shape) for k, t in a.items()}
    assert shared["k"].stride(0) == 0
    dense = {k: t.contiguous() for k, t in shared.items()}
    assert all(torch.equal(s, t) for s, t in zip(all_of(shared, dy), all_of(dense, dy)))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_a_prompt_then_tokens(mb, dtype):
    """A prompt in two pieces, then one token at a time on the state, in place: what the whole sequence gives."""
    B, L, H, K, Dk, Dv = 2, 150, 4, 2, 32, 48
    a, _ = _inputs((B, L, H, K, Dk, Dv), dtype, 31)
    wy, wh, _ = om.delta_rule(**_h(a), scale=Dk ** -0.5)
    ys, h = [], None
    for lo, hi in ((0, 77), (77, 140)):
        part = [t[:, lo:hi] for t in a.values()]
        y, h = mb.merit_delta_rule(_plan(mb, (B, hi - lo, H, K, Dk, Dv), dtype), *part, h0=h, final=True if h is None else h)
        ys.append(y)
    step = _plan(mb, (B, 1, H, K, Dk, Dv), dtype)
    for t in range(140, L):
        y, h = mb.merit_delta_rule_step(step, h, *(x[:, t] for x in a.values()), h_out=h)
        ys.append(y[:, None])
    near(torch.cat(ys, 1), wy, y_of(dtype), "y")
    near(h, wh, DELTA, "state")


def test_without_decay_and_with_total_decay(mb):
    shape = (1, 130, 2, 2, 32, 16)
    a, g = _inputs(shape, "f32", 41)
    dy, plan = g.normal(1, 130, 2, 16), _plan(mb, shape, "f32")
    y, h, st = mb.merit_delta_rule(plan, a["q"], a["k"], a["v"], None, a["beta"], final=True, states=True)
    none = dict(_h(a), g=None)
    wy, wh, _ = om.delta_rule(**none, scale=32 ** -0.5)
    near(y, wy, y_of(str(y.dtype)), "y")
    near(h, wh, DELTA, "state")
    d = mb.merit_delta_rule_backward(plan, dy, a["q"], a["k"], None, a["beta"], st)
    want = om.delta_rule_backward(host(dy), **none, scale=32 ** -0.5)
    assert d["dg"] is None
    for k in ("dq", "dk", "dv", "dbeta"):
        near(d[k], want[k], GRAD, k)
    # a decay of 0 (g = -inf): the state starts anew, and so do its gradients
    a["g"][:, 40] = a["g"][:, 100, 1] = float("-inf")
    y, h, st = mb.merit_delta_rule(plan, *a.values(), final=True, states=True)
    wy, wh, _ = om.delta_rule(**_h(a), scale=32 ** -0.5)
    near(y, wy, y_of(str(y.dtype)), "y")
    near(h, wh, DELTA, "state")
    d = mb.merit_delta_rule_backward(plan, dy, a["q"], a["k"], a["g"], a["beta"], st)
    want = om.delta_rule_backward(host(dy), **_h(a), scale=32 ** -0.5)
    for k in ("dq", "dk", "dv", "dg", "dbeta"):
        near(d[k], want[k], DECAY if k == "dg" else GRAD, k)
    y1, _ = mb.merit_delta_rule_step(_plan(mb, (1, 1, 2, 2, 32, 16), "f32"), g.normal(1, 2, 32, 16), *(t[:, 40] for t in a.values()))
    near(y1, wy[:, 40], DELTA, "token")


@pytest.mark.parametrize("L", [1, 3, 100])
def test_nothing_fades_before_the_first_token(mb, L):
    """The decay of the first token has a gradient where a state is passed in, and exactly none where it is zeros or absent."""
    shape = (2, L, 2, 1, 40, 24)
    a, g = _inputs(shape, "f32", 45)
    dy, plan = g.normal(2, L, 2, 24), _plan(mb, shape, "f32")
    h = g.normal(2, 2, 40, 24)
    h[1] = 0.0
    for h0 in (None, torch.zeros_like(h), h):
        st = mb.merit_delta_rule(plan, *a.values(), h0=h0, states=True)[-1]
        dg = mb.merit_delta_rule_backward(plan, dy, a["q"], a["k"], a["g"], a["beta"], st)["dg"]
        want = om.delta_rule_backward(host(dy), **_h(a), h0=None if h0 is None else host(h0), scale=40 ** -0.5)
        assert not dg[1, 0].any() and (h0 is h) == bool(dg[0, 0].all())
        near(dg, want["dg"], DECAY, "dg", floor=float(np.sqrt(np.mean(want["dbeta"] ** 2))))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape, lens", [((1, 1500, 1, 1, 32, 32), None), ((1, 700, 1, 1, 128, 70), None), ((1, 1025, 2, 2, 5, 9), None),
                                         ((3, 1100, 2, 1, 42, 25), [1100, 512, 130]), ((4, 1100, 1, 1, 64, 48), [0, 1, 385, 1099])])
def test_segments_of_few_sequences(mb, shape, lens, dtype):
    """Long sequences of few heads go in segments side by side: sequences that end in any of them, the last state in the first one's
    place, states kept for the backward pass, equal bits on a second call."""
    B, L, H, K, Dk, Dv = shape
    a, g = _inputs(shape, dtype, sum(shape))
    plan, h0 = _plan(mb, shape, dtype), g.normal(B, H, Dk, Dv)
    assert "merit_delta_join" in plan.kernel()
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    how = dict(lens=lens, scale=Dk ** -0.5)
    for h in (None, h0):
        wy, wh, _ = om.delta_rule(**_h(a), h0=None if h is None else host(h), **how)
        y, end = mb.merit_delta_rule(plan, *a.values(), h0=h, lens=n, final=True)
        near(y, wy, y_of(str(y.dtype)), "y")
        near(end, wh, DELTA, "state")
    again = h0.clone()
    y2, end2 = mb.merit_delta_rule(plan, *a.values(), h0=again, lens=n, final=again)
    assert end2 is again and torch.equal(y2, y) and torch.equal(end2, end)
    y3, st = mb.merit_delta_rule(plan, *a.values(), h0=h0, lens=n, states=True)
    near(y3, wy, y_of(str(y.dtype)), "y with states")
    dy = g.normal(B, L, H, Dv, dtype=TYPES[dtype][0])
    got = mb.merit_delta_rule_backward(plan, dy, a["q"], a["k"], a["g"], a["beta"], st, lens=n, dh0=True)
    want = om.delta_rule_backward(host(dy), **_h(a), h0=host(h0), **how)
    for k in ("dq", "dk", "dv", "dg", "dbeta", "dh0"):
        near(got[k], want[k], DECAY if k == "dg" else GRAD, k, floor=float(np.sqrt(np.mean(want["dbeta"] ** 2))) if k == "dg" else 0.0)


def test_segments_and_what_is_not_finite(mb):
    """A value's NaN stays in its column through later segments, a key's in its head; a decay of zero in a segment empties the state."""
    shape = (1, 1500, 2, 2, 32, 32)
    a, _ = _inputs(shape, "f32", 61)
    plan = _plan(mb, shape, "f32")
    assert "merit_delta_join" in plan.kernel()
    y, h = mb.merit_delta_rule(plan, *a.values(), final=True)
    for name in ("v", "k", "beta"):
        b = {k: t.clone() for k, t in a.items()}
        (b[name][0, 300, 0, 7:8] if name != "beta" else b[name][0, 300, 0:1]).fill_(float("nan"))
        y2, h2 = mb.merit_delta_rule(plan, *b.values(), final=True)
        assert torch.equal(y2[:, :300], y[:, :300]) and torch.equal(y2[:, :, 1], y[:, :, 1]) and torch.equal(h2[:, 1], h[:, 1])
        lost, kept = y2[0, 301:, 0], y[0, 301:, 0]
        if name == "v":
            others = [c for c in range(32) if c != 7]
            assert lost[:, 7].isnan().all() and torch.equal(lost[:, others], kept[:, others]) and h2[0, 0, :, 7].isnan().all()
        else:
            assert lost.isnan().all() and h2[0, 0].isnan().all()
    a["g"][0, 800] = float("-inf")
    y2, h2 = mb.merit_delta_rule(plan, *a.values(), final=True)
    wy, wh, _ = om.delta_rule(**_h(a), scale=32 ** -0.5)
    near(y2, wy, y_of(str(y.dtype)), "y")
    near(h2, wh, DELTA, "state")


@pytest.mark.parametrize("beta_value", [0.0, 1.0, 2.0])
def test_strengths(mb, beta_value):
    shape = (1, 100, 1, 1, 32, 16)
    a, g = _inputs(shape, "f32", 43)
    a["beta"].fill_(beta_value)
    dy, plan = g.normal(1, 100, 1, 16), _plan(mb, shape, "f32")
    y, st = mb.merit_delta_rule(plan, *a.values(), states=True)
    d = mb.merit_delta_rule_backward(plan, dy, a["q"], a["k"], a["g"], a["beta"], st)
    near(y, om.delta_rule(**_h(a), scale=32 ** -0.5)[0], y_of(str(y.dtype)), "y", floor=1e-3)
    want = om.delta_rule_backward(host(dy), **_h(a), scale=32 ** -0.5)
    for k in ("dq", "dk", "dv", "dg", "dbeta"):
        near(d[k], want[k], DECAY if k == "dg" else GRAD, k, floor=1e-3)


@pytest.mark.parametrize("same", [True, False])
def test_keys_again(mb, same):
    """Every token with the same key, or with keys of zeros: the triangular system has no zeros, or nothing but its diagonal."""
    shape = (1, 150, 1, 1, 64, 32)
    a, _ = _inputs(shape, "f32", 44)
    a["k"] = a["k"][:, :1].expand(a["k"].shape).contiguous() if same else torch.zeros_like(a["k"])
    y, h = mb.merit_delta_rule(_plan(mb, shape, "f32"), *a.values(), final=True)
    wy, wh, _ = om.delta_rule(**_h(a), scale=64 ** -0.5)
    near(y, wy, y_of(str(y.dtype)), "y", floor=1e-3)
    near(h, wh, DELTA, "state", floor=1e-3)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name, at", [("q", 70), ("k", 64), ("k", 75), ("v", 75), ("g", 75), ("beta", 75)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_behind(mb, name, at, value, dtype):
    """Tokens before it, other sequences and heads, and for v other columns, keep their bits."""
    shape = (2, 140, 4, 2, 40, 40)
    a, _ = _inputs(shape, dtype, 51)
    plan = _plan(mb, shape, dtype)
    y0, h0 = mb.merit_delta_rule(plan, *a.values(), final=True)
    a = {k: t.clone() for k, t in a.items()}
    a[name][(0, at, 1) if name in ("g", "beta") else (0, at, 1, 3)] = value
    y, h = mb.merit_delta_rule(plan, *a.values(), final=True)
    heads = [1] if name in ("v", "g", "beta") else [2, 3]
    other = [i for i in range(4) if i not in heads]
    assert torch.equal(y[1], y0[1]) and torch.equal(h[1], h0[1])
    assert torch.equal(y[0, :, other], y0[0, :, other]) and torch.equal(h[0, other], h0[0, other])
    assert torch.equal(y[0, :at], y0[0, :at])
    if name == "q":
        assert not torch.isfinite(y[0, at, heads]).any() and torch.equal(y[0, at + 1:], y0[0, at + 1:]) and torch.equal(h, h0)
    elif name == "v":
        keep = [c for c in range(40) if c != 3]
        assert torch.equal(y[0][:, :, keep], y0[0][:, :, keep]) and torch.equal(h[..., keep], h0[..., keep])
        assert not torch.isfinite(y[0, at:, 1, 3]).any() and not torch.isfinite(h[0, 1, :, 3]).any()
    else:
        assert not torch.isfinite(y[0, at:, heads]).any() and not torch.isfinite(h[0, heads]).any()


def test_empty(mb):
    """No tokens: the state goes through, gradients of nothing are nothing; no sequences: nothing to do."""
    g = Gen(5)
    plan = _plan(mb, (2, 0, 2, 1, 8, 12), "f32")
    q, v, s = torch.empty(2, 0, 1, 8, device=DEV), torch.empty(2, 0, 2, 12, device=DEV), torch.empty(2, 0, 2, device=DEV)
    h0 = g.normal(2, 2, 8, 12)
    y, h, st = mb.merit_delta_rule(plan, q, q, v, s, s, h0=h0, final=True, states=True)
    assert y.shape == (2, 0, 2, 12) and torch.equal(h, h0) and st.shape[:3] == (2, 0, 2)
    d = mb.merit_delta_rule_backward(plan, v, q, q, s, s, st, dh_last=h0, dh0=True)
    assert torch.equal(d["dh0"], h0)
    plan = _plan(mb, (0, 5, 2, 1, 8, 12), "f32")
    q, v, s = torch.empty(0, 5, 1, 8, device=DEV), torch.empty(0, 5, 2, 12, device=DEV), torch.empty(0, 5, 2, device=DEV)
    assert mb.merit_delta_rule(plan, q, q, v, s, s).shape == (0, 5, 2, 12)


def test_outputs_where_they_are_given(mb):
    """A given y between other rows, a state over the first state; memory beside them stays."""
    shape = (2, 70, 2, 2, 16, 20)
    a, g = _inputs(shape, "bf16", 61)
    plan, h0 = _plan(mb, shape, "bf16"), g.normal(2, 2, 16, 20)
    y, h = mb.merit_delta_rule(plan, *a.values(), h0=h0, final=True)
    room = torch.full((2, 70, 48), 7.0, dtype=torch.bfloat16, device=DEV)
    view = room[:, :, 5:45].unflatten(2, (2, 20))
    y2, h2 = mb.merit_delta_rule(plan, *a.values(), h0=h0, final=h0, y=view)
    assert y2 is view and h2 is h0 and torch.equal(view, y) and torch.equal(h0, h)
    assert bool((room[:, :, :5] == 7).all()) and bool((room[:, :, 45:] == 7).all())


def test_operands_refused(mb):
    shape = (1, 8, 2, 1, 16, 8)
    a, g = _inputs(shape, "f32", 71)
    plan = _plan(mb, shape, "f32")
    with pytest.raises(TypeError, match="g: expected torch.float32"):
        mb.merit_delta_rule(plan, a["q"], a["k"], a["v"], a["g"].half(), a["beta"])
    with pytest.raises(TypeError, match="q: expected torch.float32"):
        mb.merit_delta_rule(plan, a["q"].half(), a["k"], a["v"], a["g"], a["beta"])
    with pytest.raises(ValueError, match="v: expected shape"):
        mb.merit_delta_rule(plan, a["q"], a["k"], a["v"][..., :4], a["g"], a["beta"])
    with pytest.raises(ValueError, match="dimension 3 must be dense"):
        mb.merit_delta_rule(plan, a["q"], a["k"], g.normal(1, 8, 8, 2).transpose(2, 3), a["g"], a["beta"])
    with pytest.raises(TypeError, match="beta: expected a device tensor"):
        mb.merit_delta_rule(plan, a["q"], a["k"], a["v"], a["g"], None)
    with pytest.raises(mb.MeritError):
        mb.merit_delta_rule_step(mb.merit_plan_scan(mb.MERIT_F32, 1, 1, 8, 4), g.normal(1, 2, 16, 8), *(t[:, 0] for t in a.values()))
