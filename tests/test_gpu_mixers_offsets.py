"""The delta rule and the block's norms on tensors of more than 2^31 elements: rows far apart, and states behind each other.  What is
computed there has the same bits as on tensors of its own."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from token_helpers import DEV, Gen       # noqa: E402

FAR = (1 << 31) + 64            # elements from one sequence to the next


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


@pytest.fixture
def far():
    """Copies of tensors [2, L, ...] with the second sequence FAR elements behind the first, all in one piece of memory a type."""
    room, used = {}, {}

    def copy(t):
        n = t[0].numel()
        if t.dtype not in room:
            room[t.dtype], used[t.dtype] = torch.empty(FAR + (1 << 22), dtype=t.dtype, device=DEV), 0
        at = used[t.dtype]
        used[t.dtype] += -(-n // 64) * 64
        assert used[t.dtype] <= 1 << 22
        v = room[t.dtype].as_strided(t.shape, (FAR,) + t[0].contiguous().stride(), at)
        v.copy_(t)
        return v

    yield copy
    room.clear()
    torch.cuda.empty_cache()


def test_sequences_far_apart(mb, far):
    B, L, H, Dk, Dv = 2, 70, 4, 64, 40
    T, g = torch.bfloat16, Gen(1)
    q, k, v, dy = (g.normal(B, L, H, d, dtype=T) for d in (Dk, Dk, Dv, Dv))
    a, beta = -g.uniform(B, L, H, lo=0.01, hi=0.3), g.uniform(B, L, H, lo=0.1, hi=0.9)
    plan = mb.merit_plan_delta_rule(mb.MERIT_BF16, B, L, H, H, Dk, Dv)

    def run(q, k, v, a, beta, dy):
        y, h, st = mb.merit_delta_rule(plan, q, k, v, a, beta, final=True, states=True)
        return [y, h] + [t for t in mb.merit_delta_rule_backward(plan, dy, q, k, a, beta, st).values() if t is not None]

    want = run(q, k, v, a, beta, dy)
    there = [far(t) for t in (q, k, v, a, beta, dy)]
    assert all(torch.equal(s, t) for s, t in zip(run(*there), want))
    y = far(torch.zeros_like(v))
    assert mb.merit_delta_rule(plan, *there[:5], y=y) is y and torch.equal(y, want[0])
    step = mb.merit_plan_delta_rule(mb.MERIT_BF16, B, 1, H, H, Dk, Dv)
    y1 = far(torch.zeros_like(v[:, :1]))[:, 0]
    mb.merit_delta_rule_step(step, want[1], *(t[:, 3] for t in there[:5]), y=y1)
    assert torch.equal(y1, mb.merit_delta_rule_step(step, want[1], q[:, 3], k[:, 3], v[:, 3], a[:, 3], beta[:, 3])[0])


@pytest.mark.parametrize("C", [128, 770])
def test_rows_far_apart(mb, far, C):
    B, L = 2, 300
    T, g = torch.bfloat16, Gen(C)
    x, z, r, dout, dn = (g.normal(B, L, C, dtype=T) for _ in range(5))
    w = dict(after_weight=g.normal(C), scale=g.normal(C), before_weight=g.normal(C))
    plan = mb.merit_plan_block_norm(mb.MERIT_BF16, B, L, C, act=mb.MERIT_ACT_SILU)
    out, n, st = mb.merit_block_norm(plan, x, z, r, stats=True, **w)
    d = mb.merit_block_norm_backward(plan, dout, dn, x, z, r, st, dr=True, **w)
    x, z, r, dout, dn = (far(t) for t in (x, z, r, dout, dn))
    dr = far(torch.zeros_like(out))
    d2 = mb.merit_block_norm_backward(plan, dout, dn, x, z, r, st, dr=dr, **w)
    assert d2["dr"] is dr and all(torch.equal(d[k], d2[k]) for k in d if d[k] is not None)
    mb.merit_block_norm(plan, x, z, r, out=r, n=x, **w)
    assert torch.equal(r, out) and torch.equal(x, n)


def test_many_states(mb):
    """States kept of 65536 chunks and heads, 9 GB, and their gradients: the last sequences'."""
    B, few, L, H, D = 512, 8, 60, 128, 128
    T, g = torch.bfloat16, Gen(3)
    q, k, v, dy = (g.normal(few, L, H, D, dtype=T) for _ in range(4))
    a, beta = -g.uniform(few, L, H, lo=0.01, hi=0.3), g.uniform(few, L, H, lo=0.1, hi=0.9)
    dh = g.normal(few, H, D, D)

    def run(n):
        def some(t):
            return t.repeat((n // few,) + (1,) * (t.dim() - 1))

        plan = mb.merit_plan_delta_rule(mb.MERIT_BF16, n, L, H, H, D, D)
        x = [some(t) for t in (q, k, v, a, beta)]
        y, h, st = mb.merit_delta_rule(plan, *x, h0=some(dh), final=True, states=True)
        assert n == few or st.numel() > 1 << 31
        d = mb.merit_delta_rule_backward(plan, some(dy), x[0], x[1], x[3], x[4], st, dh_last=some(dh), dh0=True)
        return [t[-few:].clone() for t in (y, h, *d.values())]

    want = run(few)
    got = run(B)
    assert all(torch.equal(s, t) for s, t in zip(got, want))
    del got
    torch.cuda.empty_cache()


def test_many_states_of_single_tokens(mb):
    """131200 states of 128 x 128, 8.6 GB, in place."""
    B, few, H, D = 1025, 5, 128, 128
    g = Gen(4)
    q, k, v = (g.normal(few, H, D) for _ in range(3))
    a, beta, h = -g.uniform(few, H, lo=0.01, hi=0.3), g.uniform(few, H), g.normal(few, H, D, D)

    def run(n):
        x = [t.repeat((n // few,) + (1,) * (t.dim() - 1)) for t in (h, q, k, v, a, beta)]
        y, out = mb.merit_delta_rule_step(mb.merit_plan_delta_rule(mb.MERIT_F32, n, 1, H, H, D, D), *x, h_out=x[0])
        assert out is x[0] and (n == few or out.numel() > 1 << 31)
        return y[-few:].clone(), out[-few:].clone()

    want = run(few)
    got = run(B)
    assert all(torch.equal(s, t) for s, t in zip(got, want))
    del got
    torch.cuda.empty_cache()
