"""Group norm with an activation against the 64-bit definition, forward and backward (tolerances: token_helpers).
Chain: the sum of a group in pieces and a tree, 64 roundings; each value takes part in mean, variance and result: 256."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import tokens as ot                        # noqa: E402
from token_helpers import ACTS, DEV, TYPES, Gen, check, host, wider     # noqa: E402

CHAIN = 256


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


# N, S, C, groups: a row a group by lanes, wavefronts and workgroups; chunks of one and of many groups, of pieces of one;
# odd channel counts; one channel a group; one position; one value a group
SHAPES = [(5, 1, 64, 4), (7, 1, 1024, 16), (3, 1, 40, 8), (9, 1, 15, 3), (6, 1, 640, 1), (2, 1, 1032, 1), (5, 1, 2000, 1),
          (3, 1, 3000, 2), (2, 1, 8192, 1), (2, 1, 8200, 1), (1, 1, 9000, 1), (3, 1, 255, 1), (1000, 1, 32, 4), (1, 1, 8, 8),
          (2, 9, 64, 4), (1, 49, 96, 3), (3, 50, 40, 8), (2, 33, 15, 3), (1, 7, 2056, 1), (2, 5, 520, 2), (1, 300, 8, 8),
          (1, 40, 320, 32), (2, 1100, 40, 4), (2, 60, 60, 2), (1, 4200, 20, 1), (7, 1, 60, 6), (3, 1, 1500, 3), (2, 1000, 256, 32), (1, 2, 600, 600), (300, 2, 16, 2), (1, 4097, 3, 1)]


def _inputs(shape, dtype, seed, params=True):
    N, S, C, G = shape
    T = TYPES[dtype][0]
    g = Gen(seed)
    x = (g.normal(N, S, C) * g.uniform(C, lo=0.3, hi=2.0) + g.normal(C)).to(T)
    w, b = (g.normal(C, mean=1.0, std=0.3), g.normal(C, std=0.5)) if params else (None, None)
    return x, w, b, g.normal(N, S, C, dtype=T)


def _plan(mb, shape, dtype, act, eps=1e-5):
    return mb.merit_plan_group_norm(TYPES[dtype][1], *shape, eps, ACTS[act])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(mb, shape, dtype):
    act = ("none", "relu", "silu")[sum(shape) % 3]
    x, w, b, _ = _inputs(shape, dtype, sum(shape))
    y, mean, rstd = mb.merit_group_norm(_plan(mb, shape, dtype, act), x, w, b, stats=True)
    want = ot.group_norm(host(x), shape[3], host(w), host(b), 1e-5, act)
    for got, ref, what in zip((y, mean, rstd), want, ("y", "mean", "rstd")):
        check(got, ref, CHAIN, what)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[1] * s[2] // s[3] >= 8])
def test_backward(mb, shape, dtype):
    act = ("none", "silu")[sum(shape) % 2]
    x, w, b, dy = _inputs(shape, dtype, sum(shape) + 1)
    plan = _plan(mb, shape, dtype, act)
    _, mean, rstd = mb.merit_group_norm(plan, x, w, b, stats=True)
    got = mb.merit_group_norm_backward(plan, dy, x, mean, rstd, w, b)
    want = ot.group_norm_backward(host(dy), host(x), shape[3], host(w), host(b), 1e-5, act)
    for g, ref, what in zip(got, want, ("dx", "dw", "db")):
        check(g, ref, 4 * CHAIN, what)


@pytest.mark.parametrize("shape", [(5, 1, 64, 4), (3, 1, 15, 3), (2, 30, 64, 4)])
def test_clipped_gradient(mb, shape):
    """The clipped activation's slope jumps at 0: parameters that keep every value a tenth away from it."""
    x, _, _, dy = _inputs(shape, "f32", 11)
    plan = _plan(mb, shape, "f32", "relu")
    xh = ot.group_norm(host(x), shape[3])[0]
    b = torch.from_numpy(np.where(np.arange(shape[2]) % 2, 1.0, -1.0) * (np.abs(xh).max() + 0.1)).float().to(DEV)
    w = torch.ones(shape[2], device=DEV)
    _, mean, rstd = mb.merit_group_norm(plan, x, w, b, stats=True)
    got = mb.merit_group_norm_backward(plan, dy, x, mean, rstd, w, b)
    for g, ref, what in zip(got, ot.group_norm_backward(host(dy), host(x), shape[3], host(w), host(b), 1e-5, "relu"), "xwb"):
        check(g, ref, 4 * CHAIN, what)


@pytest.mark.parametrize("shape", [(4, 1, 64, 4), (4, 20, 64, 4)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parameters_absent_or_of_the_tensors_type(mb, shape, dtype):
    x, w, b, dy = _inputs(shape, dtype, 3)
    plan = _plan(mb, shape, dtype, "silu")
    for pw, pb in ((None, None), (w.to(x.dtype), None), (None, b.to(x.dtype)), (w.to(x.dtype), b)):
        y, mean, rstd = mb.merit_group_norm(plan, x, pw, pb, stats=True)
        check(y, ot.group_norm(host(x), shape[3], host(pw), host(pb), 1e-5, "silu")[0], CHAIN, "y")
        got = mb.merit_group_norm_backward(plan, dy, x, mean, rstd, pw, pb)
        for g, ref in zip(got, ot.group_norm_backward(host(dy), host(x), shape[3], host(pw), host(pb), 1e-5, "silu")):
            check(g, ref, 4 * CHAIN, "gradients")


@pytest.mark.parametrize("shape", [(4, 1, 64, 4), (3, 20, 64, 4), (2, 1, 30, 2)])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_slices_and_broadcasts(mb, shape, dtype):
    """Rows of a wider tensor (aligned and not), NaN beside them; one image for all; outputs in a wider tensor."""
    x, w, b, dy = _inputs(shape, dtype, 5)
    plan = _plan(mb, shape, dtype, "silu")
    y, mean, rstd = mb.merit_group_norm(plan, x, w, b, stats=True)
    dx, dw, db = mb.merit_group_norm_backward(plan, dy, x, mean, rstd, w, b)
    for front, back in ((3, 5), (8, 8), (16, 0)):
        out = wider(torch.zeros_like(x), front, back, 7.0)
        assert torch.equal(mb.merit_group_norm(plan, wider(x, front, back), w, b, y=out), out)
        ref = ot.group_norm(host(x), shape[3], host(w), host(b), 1e-5, "silu")[0]
        check(out, ref, CHAIN, "y")
        base = out._base if out._base is not None else out
        assert (base[..., :front] == 7.0).all() and (base[..., front + shape[2]:] == 7.0).all()
        got = mb.merit_group_norm_backward(plan, wider(dy, front, back), wider(x, back, front), mean, rstd, w, b)
        for g, r in zip(got, ot.group_norm_backward(host(dy), host(x), shape[3], host(w), host(b), 1e-5, "silu")):
            check(g, r, 4 * CHAIN, "gradients")
    one = x[:1].expand(shape[0], -1, -1)
    assert torch.equal(mb.merit_group_norm(plan, one, w, b), y[:1].expand(shape[0], -1, -1))


@pytest.mark.parametrize("shape", [(4, 1, 64, 4), (3, 20, 64, 4)])
def test_in_place(mb, shape):
    x, w, b, dy = _inputs(shape, "bf16", 6)
    plan = _plan(mb, shape, "bf16", "silu")
    y, mean, rstd = mb.merit_group_norm(plan, x, w, b, stats=True)
    dx, dw, db = mb.merit_group_norm_backward(plan, dy, x, mean, rstd, w, b)
    again = mb.merit_group_norm_backward(plan, dy, x, mean, rstd, w, b, dx=dy)
    assert again[0] is dy and torch.equal(dy, dx) and torch.equal(again[1], dw)
    assert torch.equal(mb.merit_group_norm(plan, x, w, b, y=x), y) and torch.equal(x, y)


@pytest.mark.parametrize("shape", [(3, 1, 256, 2), (2, 500, 32, 4), (1, 1, 4096, 1)])
def test_a_mean_far_from_zero_costs_no_digits(mb, shape):
    """Values 4096 + N(0,1) on a grid of 2^-10: exact in fp32; the mean's own rounding, 2^-12 of it, is what y may be off
    by, one in 2^12; a variance from the difference of squares would be off by 2^24 2^-24 = 1."""
    g = Gen(7)
    x = (torch.round(g.normal(*shape[:3]) * 1024) / 1024) + 4096.0
    y, mean, rstd = mb.merit_group_norm(_plan(mb, shape, "f32", "none"), x, stats=True)
    want, m, r = ot.group_norm(host(x), shape[3])
    assert np.abs(host(mean) - m).max() <= 2 * 2.0 ** -12
    np.testing.assert_allclose(host(rstd), r, rtol=1e-5)
    assert np.abs(host(y) - want).max() <= 4 * 2.0 ** -12


def test_constant_groups_and_infinities(mb):
    """No variance: rstd = 1 / sqrt(eps), y = bias.  An infinity or a NaN stays in its own group."""
    for shape in ((2, 1, 32, 4), (2, 12, 32, 4)):
        plan = _plan(mb, shape, "f32", "none", eps=1e-4)
        x, b = torch.full(shape[:3], 3.25, device=DEV), Gen(8).normal(32)
        y, mean, rstd = mb.merit_group_norm(plan, x, None, b, stats=True)
        assert torch.equal(y, b.expand_as(y)) and (mean == 3.25).all()
        np.testing.assert_allclose(host(rstd), 100.0, rtol=1e-6)
        x, w, b, _ = _inputs(shape, "f32", 9)
        clean = mb.merit_group_norm(plan, x, w, b)
        x[1, 0, 3] = float("inf")
        x[0, shape[1] - 1, 30] = float("nan")
        y = mb.merit_group_norm(plan, x, w, b)
        assert torch.isnan(y[1, 0, 3]) and torch.isnan(y[0, :, 24:]).all()
        assert torch.equal(y[1, :, 8:], clean[1, :, 8:]) and torch.equal(y[0, :, :24], clean[0, :, :24])


def test_nothing_to_do(mb):
    w = torch.ones(32, device=DEV)
    for N, S in ((0, 4), (0, 1), (3, 0)):
        plan = _plan(mb, (N, S, 32, 4), "f32", "silu")
        x = torch.empty(N, S, 32, device=DEV)
        y, mean, rstd = mb.merit_group_norm(plan, x, w, stats=True)
        assert y.shape == x.shape and (mean == 0).all()
        dx, dw, db = mb.merit_group_norm_backward(plan, x, x, mean, rstd, w)
        assert dx.shape == x.shape and (dw == 0).all() and (db == 0).all()


def test_more_images_than_an_extent_of_a_launch_holds(mb):
    shape = (70001, 2, 16, 2)
    x, w, b, dy = _inputs(shape, "f16", 10)
    plan = _plan(mb, shape, "f16", "none")
    y, mean, rstd = mb.merit_group_norm(plan, x, w, b, stats=True)
    check(y, ot.group_norm(host(x), 2, host(w), host(b))[0], CHAIN, "y")
    got = mb.merit_group_norm_backward(plan, dy, x, mean, rstd, w, b)
    for g, r in zip(got, ot.group_norm_backward(host(dy), host(x), 2, host(w), host(b))):
        check(g, r, 4 * CHAIN + 70001 // 16, "gradients")


def test_refusals(mb):
    plan = _plan(mb, (2, 3, 16, 4), "f16", "none")
    x = torch.zeros(2, 3, 16, dtype=torch.float16, device=DEV)
    with pytest.raises(TypeError, match="x: expected"):
        mb.merit_group_norm(plan, x.float())
    with pytest.raises(ValueError, match="shape"):
        mb.merit_group_norm(plan, x[:1])
    with pytest.raises(ValueError, match="dense"):
        mb.merit_group_norm(plan, x.transpose(0, 2).contiguous().transpose(0, 2))
    with pytest.raises(TypeError, match="weight"):
        mb.merit_group_norm(plan, x, torch.ones(16, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(ValueError, match="weight"):
        mb.merit_group_norm(plan, x, torch.ones(32, device=DEV)[::2])
    with pytest.raises(TypeError, match="mean"):
        mb.merit_group_norm_backward(plan, x, x, None, None)
    with pytest.raises(mb.MeritError):
        mb.merit_scan_step(plan, x, x, x, x, x, x)
