"""Selective scan against the 64-bit definition: forward, backward, single tokens (tolerances: token_helpers).
Chain: four roundings a token along the recurrence and the sum over the states: 4 L + N + 16; a gradient goes through
the recurrence twice and sums B L tokens or D channels: 3 times that, and their number."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import tokens as ot                        # noqa: E402
from token_helpers import DEV, TYPES, Gen, check, host, wider     # noqa: E402


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


# B, L, D, N, G
SHAPES = [(1, 1, 4, 16, 1), (2, 16, 64, 16, 1), (1, 17, 70, 16, 1), (2, 50, 24, 16, 3), (1, 33, 130, 16, 2), (2, 20, 9, 1, 1),
          (1, 40, 300, 1, 1), (2, 18, 10, 2, 2), (1, 35, 260, 4, 1), (2, 31, 6, 3, 1), (1, 20, 130, 8, 1), (2, 33, 12, 5, 4),
          (1, 19, 40, 13, 1), (2, 34, 33, 32, 1), (1, 16, 20, 20, 2), (2, 18, 17, 64, 1), (1, 40, 5, 50, 1), (3, 5, 16, 16, 16)]


def _inputs(shape, dtype, seed):
    B, L, D, N, G = shape
    T = TYPES[dtype][0]
    g = Gen(seed)
    return dict(x=g.normal(B, L, D, dtype=T), dt=g.normal(B, L, D, dtype=T, mean=-2.0), A=-g.uniform(D, N, lo=0.1, hi=8.0),
                B=g.normal(B, L, G, N, dtype=T), C=g.normal(B, L, G, N, dtype=T), skip=g.normal(D), z=g.normal(B, L, D, dtype=T),
                dt_bias=g.normal(D, std=0.5), h0=g.normal(B, D, N), dy=g.normal(B, L, D, dtype=T), dh=g.normal(B, D, N),
                lens=torch.from_numpy(g.rng.integers(-1, L + 2, size=B).astype(np.int32)).to(DEV))


def _plan(mb, shape, dtype, softplus=True):
    return mb.merit_plan_scan(TYPES[dtype][1], *shape, softplus)


def _few(v, names):
    return {k: v[k] for k in names}


def _ref(v, extra):
    e = {k: (t.cpu().numpy() if k == "lens" else host(t)) for k, t in extra.items() if k in ("skip", "z", "dt_bias", "h0", "lens")}
    return (host(v["x"]), host(v["dt"]), host(v["A"]), host(v["B"]), host(v["C"])), e


WAYS = [(("skip", "z", "dt_bias"), True), (("z", "h0", "lens"), True), (("skip", "dt_bias", "h0"), True), ((), False),
        (("skip", "z", "h0", "lens"), False)]


def _positive_steps(v, softplus):
    if not softplus:
        v["dt"] = v["dt"].abs() * 0.1
    return v


def _chain(shape):
    return 4 * shape[1] + shape[3] + 16


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(mb, shape, dtype):
    for names, softplus in WAYS:
        v = _positive_steps(_inputs(shape, dtype, sum(shape)), softplus)
        extra = _few(v, names)
        y, h, states = mb.merit_scan(_plan(mb, shape, dtype, softplus), v["x"], v["dt"], v["A"], v["B"], v["C"], final=True, states=True,
                                     **extra)
        args, e = _ref(v, extra)
        wy, wh, ws = ot.scan(*args, softplus=softplus, **e)
        check(y, wy, _chain(shape), "y")
        check(h, wh, _chain(shape), "h")
        h0 = e.get("h0", np.zeros_like(wh))
        for b in range(shape[0]):                       # the states before every 16th token of the sequence
            n = shape[1] if "lens" not in e else min(max(e["lens"][b], 0), shape[1])
            for k in range(-(-n // 16)):
                check(states[b, k], ws[b, 16 * k - 1] if k else h0[b], _chain(shape), "states")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(mb, shape, dtype):
    B, L, D, N, G = shape
    for names, softplus in WAYS:
        v = _positive_steps(_inputs(shape, dtype, sum(shape) + 1), softplus)
        extra = _few(v, names)
        plan = _plan(mb, shape, dtype, softplus)
        _, states = mb.merit_scan(plan, v["x"], v["dt"], v["A"], v["B"], v["C"], states=True, **extra)
        more = {k: t for k, t in extra.items() if k != "h0"}
        dh = v["dh"] if "h0" in extra else None
        got = mb.merit_scan_backward(plan, v["dy"], v["x"], v["dt"], v["A"], v["B"], v["C"], states, dh_last=dh, dh0=True, **more)
        args, e = _ref(v, extra)
        want = ot.scan_backward(host(v["dy"]), *args, dh_last=host(dh), softplus=softplus, **e)
        chain = 3 * _chain(shape)
        sums = {"dB": D // G, "dC": D // G, "dA": B * L, "dskip": B * L, "ddt_bias": B * L}
        for k, ref in want.items():
            if k in ("dz", "dskip", "ddt_bias") and k[1:] not in extra:
                assert got[k] is None, k
            else:
                check(got[k], ref, chain + sums.get(k, 0), k)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_gradient_against_differences(mb, dtype):
    """The forward kernel itself, in fp32 with h = 2^-6 and sums in 64 bits: truncation h^2 / 6 of third derivatives of
    about 1 to 10, rounding 2^-24 times the sum's size over h; both below 2 % of gradients around 1 to 10."""
    B, L, D, N, G = shape = (1, 6, 4, 3, 1)
    v = _inputs(shape, "f32", 3)
    plan = _plan(mb, shape, "f32")
    names = ("skip", "z", "dt_bias", "h0")

    def total(**new):
        u = {**v, **new}
        y, h = mb.merit_scan(plan, u["x"], u["dt"], u["A"], u["B"], u["C"], final=True, **_few(u, names))
        return float((y.double() * v["dy"].double()).sum() + (h.double() * v["dh"].double()).sum())

    _, states = mb.merit_scan(plan, v["x"], v["dt"], v["A"], v["B"], v["C"], states=True, **_few(v, names))
    got = mb.merit_scan_backward(plan, v["dy"], v["x"], v["dt"], v["A"], v["B"], v["C"], states, skip=v["skip"], z=v["z"],
                                 dt_bias=v["dt_bias"], dh_last=v["dh"], dh0=True)
    step = 2.0 ** -6
    for k in ("x", "dt", "A", "B", "C", "skip", "z", "dt_bias", "h0"):
        t, g = v[k], got["d" + k]
        num = torch.zeros(t.numel(), dtype=torch.float64)
        for i in range(t.numel()):
            up, down = t.clone(), t.clone()
            up.view(-1)[i] += step
            down.view(-1)[i] -= step
            num[i] = (total(**{k: up}) - total(**{k: down})) / (2 * step)
        d = (num - g.double().cpu().view(-1)).norm() / num.norm()
        assert d < 0.02, (k, float(d))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [16, 5, 1])
def test_a_sequence_in_parts(mb, dtype, N):
    """A prompt, its rest, then single tokens, against the whole sequence's definition; the state in place and not."""
    B, L, D, G = 2, 60, 24, 2
    v = _inputs((B, L, D, N, G), dtype, 4)
    more = _few(v, ("skip", "dt_bias"))
    args, e = _ref(v, _few(v, ("skip", "z", "dt_bias", "h0")))
    wy, wh, _ = ot.scan(*args, **e)
    ys, h, t0 = [], v["h0"].clone(), 0
    for n in (17, 32):
        part = {k: v[k][:, t0:t0 + n] for k in ("x", "dt", "B", "C", "z")}
        y, h = mb.merit_scan(_plan(mb, (B, n, D, N, G), dtype), part["x"], part["dt"], v["A"], part["B"], part["C"], z=part["z"], h0=h,
                             final=True, **more)
        ys.append(y)
        t0 += n
    plan = _plan(mb, (B, 1, D, N, G), dtype)
    for t in range(t0, L):
        y, out = mb.merit_scan_step(plan, h, v["x"][:, t], v["dt"][:, t], v["A"], v["B"][:, t], v["C"][:, t], z=v["z"][:, t],
                                    h_out=h if t % 2 else None, **more)
        assert (out is h) == bool(t % 2)
        h = out
        ys.append(y[:, None])
    check(torch.cat(ys, 1), wy, 4 * L + N + 16, "y")
    check(h, wh, 4 * L + N + 16, "h")


def test_slices_and_broadcasts(mb):
    shape = (2, 37, 24, 16, 2)
    for dtype in ("f32", "bf16"):
        v = _inputs(shape, dtype, 5)
        plan = _plan(mb, shape, dtype)
        more = _few(v, ("skip", "dt_bias"))
        y, states = mb.merit_scan(plan, v["x"], v["dt"], v["A"], v["B"], v["C"], z=v["z"], states=True, **more)
        grads = mb.merit_scan_backward(plan, v["dy"], v["x"], v["dt"], v["A"], v["B"], v["C"], states, z=v["z"], **more)
        side = wider(torch.cat([v["B"].flatten(2), v["C"].flatten(2)], 2), 3, 1)
        Bs, Cs = (t.unflatten(2, (2, 16)) for t in side.split(32, dim=2))
        xs, zs = wider(torch.cat([v["x"], v["z"]], 2), 0, 0).split(24, dim=2)
        dts = wider(v["dt"], 1, 2)
        assert torch.equal(mb.merit_scan(plan, xs, dts, v["A"], Bs, Cs, z=zs, **more), y)
        again = mb.merit_scan_backward(plan, wider(v["dy"]), xs, dts, v["A"], Bs, Cs, states, z=zs, **more)
        for k, t in grads.items():
            assert (t is None and again[k] is None) or torch.equal(t, again[k]), k
        one = mb.merit_scan(plan, v["x"][:1].expand(2, -1, -1), v["dt"][:1].expand(2, -1, -1), v["A"], v["B"][:1].expand(2, -1, -1, -1),
                            v["C"][:1].expand(2, -1, -1, -1))
        assert torch.equal(one[0], one[1])
        plan1 = _plan(mb, (2, 1, 24, 16, 2), dtype)
        a = mb.merit_scan_step(plan1, v["h0"], v["x"][:, 3], v["dt"][:, 3], v["A"], v["B"][:, 3], v["C"][:, 3], z=v["z"][:, 3], **more)
        b = mb.merit_scan_step(plan1, v["h0"], v["x"][:, 3].contiguous(), v["dt"][:, 3].contiguous(), v["A"],
                               v["B"][:, 3].contiguous(), v["C"][:, 3].contiguous(), z=v["z"][:, 3].contiguous(), **more)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("N", [16, 8, 4, 2, 5])
def test_states_that_start_anywhere(mb, N):
    """fp32 operands one element behind a 16-byte boundary, tensors of 16 bits behind an odd one."""
    def off(t):
        big = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        big[1:] = t.reshape(-1)
        return big[1:].view(t.shape)

    shape = (2, 35, 12, N, 2)
    v = _inputs(shape, "f16", 12)
    plan, plan1 = _plan(mb, shape, "f16"), _plan(mb, (2, 1, 12, N, 2), "f16")
    u = {k: off(t) for k, t in v.items()}
    names = ("skip", "z", "dt_bias", "h0", "lens")
    results = []
    for w in (v, u):
        y, h, st = mb.merit_scan(plan, w["x"], w["dt"], w["A"], w["B"], w["C"], final=True, states=True, **_few(w, names))
        g = mb.merit_scan_backward(plan, w["dy"], w["x"], w["dt"], w["A"], w["B"], w["C"], st if w is v else off(st), dh_last=w["dh"],
                                   dh0=True, **_few(w, ("skip", "z", "dt_bias", "lens")))
        s = mb.merit_scan_step(plan1, w["h0"], off(w["x"][:, 0]), off(w["dt"][:, 0]), w["A"], off(w["B"][:, 0]), off(w["C"][:, 0]),
                               h_out=off(w["h0"]))
        results.append([y, h, *g.values(), *s])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_what_lies_behind_an_end_is_not_read(mb):
    shape = (5, 40, 20, 16, 1)
    v = _inputs(shape, "f32", 6)
    ends = (0, 1, 16, 17, 40)
    lens = torch.tensor(ends, dtype=torch.int32, device=DEV)
    plan = _plan(mb, shape, "f32")
    d = {k: v[k].clone() for k in ("x", "dt", "B", "C", "z", "dy")}
    for b, n in enumerate(ends):
        for k, t in d.items():
            t[b, n:] = float("nan") if k in ("x", "B", "dy") else float("inf")
    kw = dict(skip=v["skip"], dt_bias=v["dt_bias"], lens=lens)
    y, h, st = mb.merit_scan(plan, v["x"], v["dt"], v["A"], v["B"], v["C"], z=v["z"], h0=v["h0"], final=True, states=True, **kw)
    y2, h2, st2 = mb.merit_scan(plan, d["x"], d["dt"], v["A"], d["B"], d["C"], z=d["z"], h0=v["h0"], final=True, states=True, **kw)
    assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(h[0], v["h0"][0]) and (y[0] == 0).all()
    a = mb.merit_scan_backward(plan, v["dy"], v["x"], v["dt"], v["A"], v["B"], v["C"], st, z=v["z"], dh_last=v["dh"], dh0=True, **kw)
    b = mb.merit_scan_backward(plan, d["dy"], d["x"], d["dt"], v["A"], d["B"], d["C"], st2, z=d["z"], dh_last=v["dh"], dh0=True, **kw)
    for k in a:
        assert torch.equal(a[k], b[k]), k
    assert torch.equal(a["dh0"][0], v["dh"][0])


def test_infinities_keep_to_their_channel(mb):
    """An infinite input, with states that are and are not a multiple of four, and a channel that does not fill a wavefront."""
    for N in (16, 5, 3, 1):
        shape = (1, 20, 10, N, 1)
        v = _inputs(shape, "f32", 7)
        plan = _plan(mb, shape, "f32")
        clean = mb.merit_scan(plan, v["x"], v["dt"], v["A"], v["B"].abs(), v["C"].abs())
        x = v["x"].clone()
        x[0, 7, 4] = float("inf")
        y = mb.merit_scan(plan, x, v["dt"], v["A"], v["B"].abs(), v["C"].abs())
        assert torch.isinf(y[0, 7:, 4]).all(), N
        y[0, 7:, 4] = clean[0, 7:, 4]
        assert torch.equal(y, clean), N


def test_steps_far_out(mb):
    """Steps from next to nothing to large ones: log(1 + exp(v)) keeps its digits, decays reach 0 and 1."""
    B, L, D, N = 1, 32, 8, 4
    v = _inputs((B, L, D, N, 1), "f32", 8)
    v["dt"] = torch.linspace(-60, 60, B * L * D, device=DEV).view(B, L, D)
    v["x"] = v["x"] / torch.nn.functional.softplus(v["dt"].double()).float()       # (inputs of about 1 whatever the step)
    y, h = mb.merit_scan(_plan(mb, (B, L, D, N, 1), "f32"), v["x"], v["dt"], v["A"], v["B"], v["C"], final=True)
    args, e = _ref(v, {})
    wy, wh, _ = ot.scan(*args)
    check(y, wy, 4 * L + 64, "y")
    check(h, wh, 4 * L + 64, "h")


def test_nothing_to_do(mb):
    for B, L in ((0, 5), (2, 0)):
        v = _inputs((B, L, 8, 4, 1), "f32", 9)
        plan = _plan(mb, (B, L, 8, 4, 1), "f32")
        y, h, st = mb.merit_scan(plan, v["x"], v["dt"], v["A"], v["B"], v["C"], h0=v["h0"], final=True, states=True)
        assert y.shape == v["x"].shape and torch.equal(h, v["h0"])
        g = mb.merit_scan_backward(plan, v["dy"], v["x"], v["dt"], v["A"], v["B"], v["C"], st, skip=v["skip"], dh_last=v["dh"], dh0=True)
        assert (g["dA"] == 0).all() and (g["dskip"] == 0).all() and torch.equal(g["dh0"], v["dh"])


def test_offsets_past_32_bits(mb):
    """Rows 2^27 elements apart, of inputs and of the result."""
    B, L, D, N = shape = (1, 36, 16, 16)
    v = _inputs(shape + (1,), "f16", 10)
    plan = _plan(mb, shape + (1,), "f16")
    y = mb.merit_scan(plan, v["x"], v["dt"], v["A"], v["B"], v["C"])
    big = torch.empty((L - 1) * (1 << 27) + 4096, dtype=torch.float16, device=DEV)
    far = {}
    for i, k in enumerate(("x", "dt", "B", "C")):
        t = v[k]
        far[k] = big[512 * i:].as_strided(t.shape, (0, 1 << 27) + t.stride()[2:])
        far[k].copy_(t)
    out = big[2048:].as_strided((B, L, D), (0, 1 << 27, 1))
    mb.merit_scan(plan, far["x"], far["dt"], v["A"], far["B"], far["C"], y=out)
    assert torch.equal(out, y)


def test_refusals(mb):
    shape = (2, 5, 8, 4, 2)
    v = _inputs(shape, "f16", 11)
    plan = _plan(mb, shape, "f16")
    ok = [v["x"], v["dt"], v["A"], v["B"], v["C"]]
    for i, bad, err in ((0, v["x"].float(), TypeError), (2, v["A"].half(), TypeError), (2, v["A"].t().contiguous().t(), ValueError),
                        (3, v["B"][:, :, :1], ValueError), (4, v["C"].transpose(2, 3).contiguous().transpose(2, 3), ValueError),
                        (1, v["dt"].cpu(), TypeError), (1, None, TypeError)):
        args = list(ok)
        args[i] = bad
        with pytest.raises(err):
            mb.merit_scan(plan, *args)
    with pytest.raises(ValueError, match="h0"):
        mb.merit_scan(plan, *ok, h0=v["h0"].transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(TypeError, match="states"):
        mb.merit_scan_backward(plan, v["dy"], *ok, None)
    with pytest.raises(mb.MeritError):
        mb.merit_causal_conv(plan, v["x"], v["A"])
