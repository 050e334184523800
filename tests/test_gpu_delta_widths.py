"""The delta rule where a workgroup takes 32 and 64 columns of v from chunk to chunk, in one slice and several, all of its wavefronts
with columns, in one piece and in segments (tolerances: mixer_helpers).  Sequences times heads choose the columns: as few as leave
no compute unit a second workgroup."""
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


def _whole(mb, shape, dtype, lens=None, front=None, segments=False):
    """Forward without and with states, backward with gradients of both states, against the definition.  front: q, k, v and dy are slices
    that far into wider rows."""
    B, L, H, K, Dk, Dv = shape
    T, g = TYPES[dtype][0], Gen(sum(shape))

    def rows(*s, **kw):
        t = g.normal(*s, dtype=T, **kw)
        return t if front is None else wider(t.flatten(2), front).unflatten(2, s[2:])

    q, k, v, dy = rows(B, L, K, Dk), rows(B, L, K, Dk), rows(B, L, H, Dv), rows(B, L, H, Dv)
    a, beta = -torch.exp(g.uniform(B, L, H, lo=-6.0, hi=0.0)), g.uniform(B, L, H, lo=0.05, hi=0.95)
    h0, dh = g.normal(B, H, Dk, Dv), g.normal(B, H, Dk, Dv)
    plan = mb.merit_plan_delta_rule(TYPES[dtype][1], *shape)
    assert ("chunks+merit_delta_join" in plan.kernel()) == segments
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    ins, how = [host(t) for t in (q, k, v, a, beta)], dict(h0=host(h0), lens=lens, scale=Dk ** -0.5)
    wy, wh, _ = om.delta_rule(*ins, **how)
    y, h = mb.merit_delta_rule(plan, q, k, v, a, beta, h0=h0, lens=n, final=True)
    y2, h2, states = mb.merit_delta_rule(plan, q, k, v, a, beta, h0=h0, lens=n, final=True, states=True)
    for got in (y, y2):
        near(got, wy, y_of(str(y.dtype)), "y")
    for got in (h, h2):
        near(got, wh, DELTA, "state")
    got = mb.merit_delta_rule_backward(plan, dy, q, k, a, beta, states, lens=n, dh_last=dh, dh0=True)
    want = om.delta_rule_backward(host(dy), *ins, dh_last=host(dh), **how)
    for name, w in want.items():
        near(got[name], w, DECAY if name == "dg" else GRAD, name, floor=float(np.sqrt(np.mean(want["dbeta"] ** 2))) if name == "dg" else 0.0)


# 32 columns (64 heads and sequences of 96); 64 in one slice and in three, the last with two columns, for keys of up to 32, 64 and 128
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape, front", [((16, 130, 4, 2, 128, 96), None), ((16, 70, 4, 4, 20, 96), None), ((4, 70, 13, 13, 128, 130), None),
                                          ((4, 66, 13, 13, 100, 130), 3), ((6, 100, 44, 22, 64, 64), 8), ((5, 129, 60, 20, 30, 100), None),
                                          ((6, 70, 44, 44, 90, 64), 1)])
def test_wider_tiles(mb, shape, front, dtype):
    _whole(mb, shape, dtype, front=front)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_wider_tiles_of_short_sequences(mb, dtype):
    _whole(mb, (8, 140, 33, 11, 72, 64), dtype, lens=[0, 1, 63, 64, 65, 128, 139, 140])


# the transitions' columns in slices of their own behind those of v, 32 and 64 wide, and segments' results as wide
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape, lens, front", [((1, 900, 8, 4, 65, 130), None, None), ((1, 1100, 16, 8, 128, 70), None, 8),
                                                ((1, 1100, 16, 4, 40, 72), None, None), ((1, 1100, 16, 4, 72, 72), None, None),
                                                ((1, 1100, 24, 8, 72, 50), None, 3), ((2, 1000, 8, 8, 64, 66), [1000, 449], None),
                                                ((3, 1000, 6, 6, 32, 96), [1, 999, 512], None)])
def test_wider_tiles_in_segments(mb, shape, lens, front, dtype):
    _whole(mb, shape, dtype, lens=lens, front=front, segments=True)
