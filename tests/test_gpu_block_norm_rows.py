"""The norms before and after a block where a workgroup takes many rows one after the other, and their forms at the longest rows, against
the 64-bit definition (tolerances: mixer_helpers)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from mixer_helpers import NORM, near                    # noqa: E402
from test_gpu_block_norm import NAMES, _case, _check, _plan, _want     # noqa: E402
from token_helpers import Gen                           # noqa: E402


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


# Several times the rows that all workgroups have at once (by runs of lanes 64 to 1024 wavefronts of four with 1 to 64 rows each, else
# up to 1024 workgroups of 256 threads or 512 of 512): sequences shorter than the way to the next row, so that it crosses ends, and longer ones
ROWS = [(70, 600, 128), (9000, 7, 24), (3, 19000, 37), (3, 1700, 1024), (700, 7, 770), (2, 1300, 4100), (521, 5, 4104), (3, 700, 2051)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", ["after gate:silu scale stream before", "after gate:sigmoid layer scale stream before f32", "after gate:none"])
@pytest.mark.parametrize("shape", ROWS)
def test_many_rows_a_workgroup(mb, shape, form, dtype):
    _check(mb, shape, dtype, form)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(70, 600, 128), (3, 1700, 1024), (521, 5, 4104)])
def test_many_rows_in_place_and_strided(mb, shape, dtype):
    """Rows between other rows, one row of gates for a sequence, results over their operands: the same bits as apart and dense."""
    x, z, r, vec, kw, dout, dn, R = _case(shape, dtype, "after gate:silu scale stream before", 5)
    plan = _plan(mb, shape, dtype, kw, R)
    z = z[:, :1].expand(shape)
    out, n, st = mb.merit_block_norm(plan, x, z.contiguous(), r, **vec, stats=True)
    d = mb.merit_block_norm_backward(plan, dout, dn, x, z.contiguous(), r, st, dr=True, **vec)
    apart = [torch.stack([t, torch.full_like(t, float("nan"))], 2).flatten(1, 2)[:, ::2] for t in (x, r, dout, dn)]
    sx, sr, sdout, sdn = apart
    o2, n2, st2 = mb.merit_block_norm(plan, sx, z, sr, **vec, stats=True)
    assert torch.equal(o2, out) and torch.equal(n2, n)
    assert all(s is t is None or torch.equal(s, t) for s, t in zip(st, st2))
    d2 = mb.merit_block_norm_backward(plan, sdout, sdn, sx, z, sr, st, dr=sdout, **vec)
    assert d2["dr"] is sdout and all(torch.equal(d[k], d2[k]) for k in d if d[k] is not None)
    o3, n3 = mb.merit_block_norm(plan, sx, z, sr, **vec, out=sr, n=sx)
    assert o3 is sr and n3 is sx and torch.equal(o3, out) and torch.equal(n3, n)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("C", [2048, 4094, 4096, 8188, 8190, 8191, 8192])
@pytest.mark.parametrize("form", ["after stream before", "after gate:silu", "stream before f32"])
def test_forms_of_the_longest_rows(mb, form, C, dtype):
    _check(mb, (2, 3, C), dtype, form)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layer, biases", [(False, True), (True, False)])
@pytest.mark.parametrize("shape", [(2, 21, 48), (2, 13, 640), (1, 7, 2050), (1, 3, 8192)])
def test_biases_without_means_and_means_without_biases(mb, shape, layer, biases, dtype):
    x, z, r, vec, kw, dout, dn, R = _case(shape, dtype, "after gate:silu scale stream before" + " layer" * layer, sum(shape))
    g = Gen(sum(shape) + 1)
    for name in ("after_bias", "before_bias"):
        vec[name] = g.normal(shape[2], std=0.5) if biases else None
    plan = _plan(mb, shape, dtype, kw, R)
    out, n, stats = mb.merit_block_norm(plan, x, z, r, **vec, stats=True)
    (wo, wn), wg = _want(x, z, r, vec, kw, dout, dn)
    near(out, wo, NORM, "out")
    near(n, wn, NORM, "n")
    d = mb.merit_block_norm_backward(plan, dout, dn, x, z, r, stats, dr=True, **vec)
    for k, got in d.items():
        assert (got is None) == (k[1:] in NAMES and vec[k[1:]] is None), k
        if got is not None:
            near(got, wg[k], 4 * NORM, k)
