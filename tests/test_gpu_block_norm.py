"""The norms before and after a block against the 64-bit definition, forward and backward (tolerances: mixer_helpers)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from mixer_helpers import NORM, near                    # noqa: E402
from oracle import mixers as om                         # noqa: E402
from token_helpers import DEV, TYPES, Gen, host, wider  # noqa: E402

NAMES = ("after_weight", "after_bias", "scale", "before_weight", "before_bias")


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


# B, L, C: rows by runs of lanes, by workgroups of 256 and 512 threads, of 1 to 16 vectors a thread; vectors of 16 bytes, two values, one
SHAPES = [(1, 1, 1), (2, 3, 8), (3, 70, 64), (2, 33, 130), (1, 5, 96), (5, 7, 37), (2, 9, 512), (3, 11, 770), (2, 5, 1025), (1, 3, 2048),
          (2, 3, 2051), (1, 4, 4096), (1, 3, 5000), (2, 2, 8192), (1, 3, 8191), (2, 3, 8190), (3, 5, 7000), (1, 2, 4094), (700, 3, 24), (1, 1500, 256)]
# which parts there are: norm after, gate, its function, scale, stream, norm before, layer norm, fp32 stream
FORMS = [("after gate:silu", {}), ("after stream before", {}), ("after scale stream before layer", {}), ("stream before f32", {}),
         ("after gate:none scale stream f32", {}), ("gate:sigmoid scale stream before layer f32", {}), ("after layer before", {}),
         ("after gate:relu stream before", {})]


def _case(shape, dtype, form, seed):
    B, L, C = shape
    words = form.split()
    T, g = TYPES[dtype][0], Gen(seed)
    R = torch.float32 if "f32" in words else T
    act = next((w.split(":")[1] for w in words if w.startswith("gate")), None)
    after, before, layer = ("after" in words), ("before" in words), ("layer" in words)
    x = (g.normal(B, L, C) * g.uniform(C, lo=0.5, hi=2.0) + g.normal(C, std=0.3)).to(T)
    z = None
    if act:         # (the clipped gate's slope jumps at 0: values that keep away from it)
        z = g.normal(B, L, C)
        z = (z + 0.1 * torch.sign(z)).to(T)
    r = g.normal(B, L, C, dtype=R, std=2.0) if "stream" in words else None
    vec = {"after_weight": g.normal(C, mean=1.0, std=0.3) if after else None,
           "after_bias": g.normal(C, std=0.5) if after and layer else None,
           "scale": g.normal(C, std=0.3).to(T) if "scale" in words else None,
           "before_weight": g.normal(C, mean=1.0, std=0.3).to(T) if before else None,
           "before_bias": g.normal(C, std=0.5) if before and layer else None}
    kw = dict(layer=layer, act=act or "none", after=after, before=before)
    dout = g.normal(B, L, C, dtype=R) if "stream" in words or not before else None
    dn = g.normal(B, L, C, dtype=T) if before else None
    return x, z, r, vec, kw, dout, dn, R


def _plan(mb, shape, dtype, kw, R, eps=1e-5):
    act = {"none": mb.MERIT_ACT_NONE, "relu": mb.MERIT_ACT_RELU, "silu": mb.MERIT_ACT_SILU, "sigmoid": mb.MERIT_ACT_SIGMOID}[kw["act"]]
    return mb.merit_plan_block_norm(TYPES[dtype][1], *shape, stream=mb.MERIT_F32 if R == torch.float32 else TYPES[dtype][1],
                                    layer=kw["layer"], eps=eps, act=act, after=kw["after"], before=kw["before"])


def _h(t):
    return None if t is None else host(t)


def _want(x, z, r, vec, kw, dout=None, dn=None, eps=1e-5):
    v = dict(zip(("aw", "ab", "scale", "bw", "bb"), (_h(vec[n]) for n in NAMES)))
    out = om.block_norm(_h(x), _h(z), _h(r), **v, eps=eps, **kw)
    if dout is None and dn is None:
        return out
    return out, om.block_norm_backward(_h(dout), _h(dn), _h(x), _h(z), _h(r), **v, eps=eps, **kw)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(mb, shape, dtype):
    form = FORMS[sum(shape) % len(FORMS)][0]
    if shape[2] < 8 and "layer" in form:
        form = FORMS[1][0]              # (a layer norm of one value is 0)
    _check(mb, shape, dtype, form)


@pytest.mark.parametrize("form", [f for f, _ in FORMS])
@pytest.mark.parametrize("shape", [(2, 21, 48), (2, 13, 640)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_form(mb, form, shape, dtype):
    _check(mb, shape, dtype, form)


def _check(mb, shape, dtype, form):
    x, z, r, vec, kw, dout, dn, R = _case(shape, dtype, form, sum(shape))
    plan = _plan(mb, shape, dtype, kw, R)
    out, n, stats = mb.merit_block_norm(plan, x, z, r, **vec, stats=True)
    (wo, wn), wg = _want(x, z, r, vec, kw, dout, dn)
    near(out, wo, NORM, "out")
    assert (n is None) == (wn is None)
    if n is not None:
        near(n, wn, NORM, "n")
    d = mb.merit_block_norm_backward(plan, dout, dn, x, z, r, stats, dr=r is not None, **vec)
    for k, got in d.items():
        if got is None:
            assert k == "dz" and z is None or k == "dr" and r is None or k[1:] in NAMES and vec[k[1:]] is None, k
            continue
        # (of rows of few values next to nothing is left of dx, which is a difference of values of the size of dr)
        near(got, wg[k], 4 * NORM, k, floor=float((wg["dr"] ** 2).mean() ** 0.5) if shape[2] < 8 else 0.0)
    plain = mb.merit_block_norm(plan, x, z, r, **vec)
    assert torch.equal(plain[0], out) and (n is None or torch.equal(plain[1], n))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [64, 61, 1000, 2048])
def test_views_and_a_gate_a_sequence(mb, C, dtype):
    """Slices of wider rows off every alignment, rows between other rows, one row of gates for a sequence: the same bits."""
    shape = (3, 9, C)
    x, z, r, vec, kw, dout, dn, R = _case(shape, dtype, "after gate:silu scale stream before", C)
    plan = _plan(mb, shape, dtype, kw, R)
    z = z[:, :1].expand(shape)

    def all_of(x, z, r, dout, dn):
        out, n, st = mb.merit_block_norm(plan, x, z, r, **vec, stats=True)
        return [out, n] + [t for t in mb.merit_block_norm_backward(plan, dout, dn, x, z, r, st, dr=True, **vec).values() if t is not None]

    want = all_of(x, z.contiguous(), r, dout, dn)
    assert z.stride(1) == 0
    assert all(torch.allclose(s.float(), t.float(), rtol=0, atol=0) for s, t in zip(all_of(x, z, r, dout, dn), want))
    odd = [wider(t) for t in (x, z.contiguous(), r, dout, dn)]
    # (another width of loads: the sums over a row go in another order)
    for s, t in zip(all_of(*odd), want):
        near(s, host(t), 4 * NORM, "slices")
    even = [torch.stack([t, torch.full_like(t, float("nan"))], 2).flatten(1, 2)[:, ::2] for t in (x, z.contiguous(), r, dout, dn)]
    assert all(torch.equal(s, t) for s, t in zip(all_of(*even), want))


def test_in_place(mb):
    """The stream over itself, the next block's input over x, the stream's gradient over its own."""
    shape = (2, 30, 256)
    x, z, r, vec, kw, dout, dn, R = _case(shape, "bf16", "after gate:silu scale stream before f32", 3)
    plan = _plan(mb, shape, "bf16", kw, R)
    out, n, st = mb.merit_block_norm(plan, x, z, r, **vec, stats=True)
    d = mb.merit_block_norm_backward(plan, dout, dn, x, z, r, st, dr=True, **vec)
    d2 = mb.merit_block_norm_backward(plan, dout, dn, x, z, r, st, dr=dout, **vec)
    assert d2["dr"] is dout and all(torch.equal(d[k], d2[k]) for k in d if d[k] is not None)
    o2, n2 = mb.merit_block_norm(plan, x, z, r, **vec, out=r, n=x)
    assert o2 is r and n2 is x and torch.equal(o2, out) and torch.equal(n2, n)


def test_far_means_and_tiny_rows(mb):
    """A layer norm of values round 1000 keeps their differences; rows of zeros give zeros; nothing overflows in a square's sum."""
    shape = (1, 40, 512)
    g = Gen(8)
    plan = mb.merit_plan_block_norm(mb.MERIT_F32, *shape, layer=True, eps=1e-5, before=False)
    x = g.normal(*shape, mean=1000.0)
    near(mb.merit_block_norm(plan, x)[0], om.block_norm(host(x), layer=True, eps=1e-5, before=False)[0], NORM * 1000, "far")
    plan = mb.merit_plan_block_norm(mb.MERIT_BF16, *shape, before=False)
    x = torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
    x[0, 1] = 2.0 ** 40
    y = mb.merit_block_norm(plan, x)[0]
    assert not y[0, 0].any() and torch.equal(y[0, 1], torch.ones_like(y[0, 1]))


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_rows_keep_to_themselves(mb, value):
    for C in (24, 300):
        shape = (1, 20, C)
        x, z, r, vec, kw, dout, dn, R = _case(shape, "f32", "after gate:silu stream before", 4)
        plan = _plan(mb, shape, "f32", kw, R)
        o0, n0 = mb.merit_block_norm(plan, x, z, r, **vec)
        x = x.clone()
        x[0, 7, 5] = value
        o, n = mb.merit_block_norm(plan, x, z, r, **vec)
        rest = [i for i in range(20) if i != 7]
        assert torch.equal(o[:, rest], o0[:, rest]) and torch.equal(n[:, rest], n0[:, rest])
        assert not torch.isfinite(o[0, 7, 5]) and torch.isnan(n[0, 7]).any()


def test_empty(mb):
    for shape in ((0, 3, 16), (2, 0, 16)):
        plan = mb.merit_plan_block_norm(mb.MERIT_F32, *shape)
        x, w = torch.empty(shape, device=DEV), torch.ones(16, device=DEV)
        out, n, st = mb.merit_block_norm(plan, x, None, x, after_weight=w, before_weight=w, stats=True)
        assert out.shape == shape and n.shape == shape
        d = mb.merit_block_norm_backward(plan, x, x, x, None, x, st, dr=True, after_weight=w, before_weight=w)
        assert not d["dafter_weight"].any() and not d["dbefore_weight"].any() and d["dx"].shape == shape


def test_operands_refused(mb):
    plan = mb.merit_plan_block_norm(mb.MERIT_BF16, 1, 4, 16, stream=mb.MERIT_F32, before=False)
    x, w = torch.zeros(1, 4, 16, dtype=torch.bfloat16, device=DEV), torch.ones(16, device=DEV)
    with pytest.raises(TypeError, match="r: expected torch.float32"):
        mb.merit_block_norm(plan, x, None, x)
    with pytest.raises(mb.MeritError):
        mb.merit_block_norm(plan, x, before_weight=w)        # a weight of a norm that the plan does not have
    with pytest.raises(ValueError, match="expected shape"):
        mb.merit_block_norm(plan, x, x[:, :, :8])
    with pytest.raises(mb.MeritError):
        mb.merit_block_norm_backward(plan, None, x, x, None, None, (None,) * 4)
    with pytest.raises(mb.MeritError):
        mb.merit_block_norm(mb.merit_plan_group_norm(mb.MERIT_BF16, 1, 4, 16, 1), x)
