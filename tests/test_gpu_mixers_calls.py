"""How the delta rule and the block's norms are called: the same bits every time, through the native module and through ctypes,
on other streams, under stream capture; memory that a call hands back; a run of them as a model makes it."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from mixer_helpers import GRAD, NORM, near      # noqa: E402
from token_helpers import DEV, TYPES, Gen, host     # noqa: E402


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


def _block(mb, dtype="bf16", B=2, L=150, H=4, K=2, Dk=64, Dv=40, seed=1):
    """A block: the rule over heads, a gated norm of each head's result, the sum with the residual stream and the next norm, all
    forward and backward, and a token more: a function of the stream argument, which returns all results."""
    T, code, _ = TYPES[dtype]
    g = Gen(seed)
    q, k, v = g.normal(B, L, K, Dk, dtype=T), g.normal(B, L, K, Dk, dtype=T), g.normal(B, L, H, Dv, dtype=T)
    a, beta = -g.uniform(B, L, H, lo=0.01, hi=0.5), g.uniform(B, L, H)
    z, r, dn = g.normal(B, L, H * Dv, dtype=T), g.normal(B, L, H * Dv), g.normal(B, L, H * Dv, dtype=T)
    w, wa, wb, s = g.normal(Dv), g.normal(H * Dv), g.normal(H * Dv), g.normal(H * Dv)
    rule = mb.merit_plan_delta_rule(code, B, L, H, K, Dk, Dv)
    heads = mb.merit_plan_block_norm(code, B * L, H, Dv, act=mb.MERIT_ACT_SILU, before=False)
    end = mb.merit_plan_block_norm(code, B, L, H * Dv, stream=mb.MERIT_F32)

    def run(**kw):
        y, h, st = mb.merit_delta_rule(rule, q, k, v, a, beta, final=True, states=True, **kw)
        rows, gates = y.view(B * L, H, Dv), z.view(B * L, H, Dv)
        o, _, hs = mb.merit_block_norm(heads, rows, gates, after_weight=w, stats=True, **kw)
        x = o.view(B, L, H * Dv)
        out, n, es = mb.merit_block_norm(end, x, None, r, after_weight=wa, scale=s, before_weight=wb, stats=True, **kw)
        d = mb.merit_block_norm_backward(end, r, dn, x, None, r, es, dr=True, after_weight=wa, scale=s, before_weight=wb, **kw)
        dh = mb.merit_block_norm_backward(heads, d["dx"].view(B * L, H, Dv), None, rows, gates, None, hs, after_weight=w, **kw)
        dd = mb.merit_delta_rule_backward(rule, dh["dx"].view(B, L, H, Dv), q, k, a, beta, st, dh0=True, **kw)
        y1, h1 = mb.merit_delta_rule_step(rule, h, q[:, 3], k[:, 3], v[:, 3], a[:, 3], beta[:, 3], **kw)
        return [y, h, st, o, out, n, y1, h1] + [t for r_ in (d, dh, dd) for t in r_.values() if t is not None]

    run.inputs = dict(q=q, k=k, v=v, g=a, beta=beta, z=z, r=r, dn=dn, w=w, wa=wa, wb=wb, s=s)
    return run


def _bytes(t):
    return t.contiguous().view(torch.uint8)


def _same(a, b):
    """The same bits (what the delta rule keeps for its backward pass holds 16-bit numbers, which are not all numbers as fp32)"""
    return len(a) == len(b) and all(torch.equal(_bytes(s), _bytes(t)) for s, t in zip(a, b))


def test_the_same_bits_every_time_and_by_either_way(mb, monkeypatch):
    run = _block(mb)
    first = run()
    torch.cuda.synchronize()
    for _ in range(3):
        assert _same(run(), first)
    from paper_1911_03458_amd import tokens
    called = []
    general = tokens._general
    monkeypatch.setattr(tokens, "_general", lambda *a: called.append(a[1]) or general(*a))
    assert _same(run(), first) and not called            # (the native module took every call)
    monkeypatch.setattr(mb, "_calls", False)
    run2 = _block(mb)                                    # plans that have not met the module
    assert _same(run2(), first) and len(called) == 7


def test_on_another_stream(mb):
    run = _block(mb)
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = run(stream=side)
    with torch.cuda.stream(side):
        b = run()
        c = run(stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert _same(a, want) and _same(b, want) and _same(c, want)


def test_two_streams_at_once(mb):
    """One plan, two calls in flight: each has scratch memory of its own."""
    run = _block(mb, B=4, L=700)
    want = run()
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(3):
        for side in sides:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                got.append(run())
    torch.cuda.synchronize()
    assert all(_same(g, want) for g in got)


def test_under_capture(mb):
    """Recorded once, replayed between the program's own work: every replay as the eager call."""
    run = _block(mb)
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out))
    for i in range(4):
        for graph, out in graphs:
            for t in out:
                t.fill_(float(i))
            torch.randn(1000, device=DEV).sum().item()
            graph.replay()
            torch.cuda.synchronize()
            assert _same(out, want), i


def test_segments_under_capture_and_on_two_streams(mb):
    """A long sequence in segments, its last state in place of the first: two graphs and two streams, each with scratch memory of its
    own, and every replay as the eager call."""
    g, B, L, H, D = Gen(71), 1, 1500, 2, 48
    plan = mb.merit_plan_delta_rule(mb.MERIT_F32, B, L, H, H, D, D)
    assert "merit_delta_join" in plan.kernel()
    inputs = [(g.normal(B, L, H, D), g.normal(B, L, H, D), g.normal(B, L, H, D), -g.uniform(B, L, H, lo=0.0, hi=0.1),
               g.uniform(B, L, H, lo=0.1, hi=0.9)) for _ in range(2)]
    first = g.normal(B, H, D, D)

    def run(i, h):
        return mb.merit_delta_rule(plan, *inputs[i], h0=h, final=h)

    want = [run(i, first.clone()) for i in range(2)]
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(3):
        for i, side in enumerate(streams):
            with torch.cuda.stream(side):
                got.append((i, run(i, first.clone())))
    torch.cuda.synchronize()
    assert all(_same(out, want[i]) for i, out in got)
    graphs = []
    for i in range(2):
        graph, h = torch.cuda.CUDAGraph(), first.clone()
        with torch.cuda.graph(graph):
            out = run(i, h)
        graphs.append((graph, out, h))
    for _ in range(3):
        for i, (graph, out, h) in enumerate(graphs):
            h.copy_(first)
            torch.randn(1000, device=DEV).sum().item()
            graph.replay()
            torch.cuda.synchronize()
            assert _same(out, want[i])


def test_scratch_memory_is_handed_back(mb):
    run = _block(mb)
    run()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    out = run()
    del out
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == before


def test_a_block_and_its_gradients(mb):
    """The whole run in fp32 against torch's own derivatives of the formulas in 64 bits."""
    run = _block(mb, "f32", B=1, L=70, H=2, K=1, Dk=16, Dv=24)
    got = run()
    p = {k: t.double().requires_grad_() for k, t in run.inputs.items() if k != "dn"}
    B, L, H, Dv = p["v"].shape

    def unit(x):
        return x / torch.sqrt((x * x).sum(-1, keepdim=True) + 1e-6)

    def rms(x, eps=1e-6):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)

    q, k = (unit(p[n]).repeat_interleave(H, dim=2) for n in "qk")
    S, ys = torch.zeros(B, H, 16, Dv, dtype=torch.float64, device=DEV), []
    for t in range(L):
        S = S * torch.exp(p["g"][:, t])[..., None, None]
        u = p["beta"][:, t, :, None] * (p["v"][:, t] - (S * k[:, t, :, :, None]).sum(2))
        S = S + k[:, t, :, :, None] * u[:, :, None]
        ys.append((S * q[:, t, :, :, None]).sum(2) / 4)
    y = torch.stack(ys, 1)
    o = rms(y) * p["w"] * torch.nn.functional.silu(p["z"].view(B, L, H, Dv))
    out = p["r"] + p["s"] * rms(o.view(B, L, -1)) * p["wa"]
    n = rms(out) * p["wb"]
    loss = (out * run.inputs["r"].double()).sum() + (n * run.inputs["dn"].double()).sum()
    grads = torch.autograd.grad(loss, [p[k] for k in ("q", "k", "v", "g", "beta", "z", "r", "w", "wa", "wb", "s")])
    want = dict(zip(("q", "k", "v", "g", "beta", "z", "r", "w", "wa", "wb", "s"), grads))
    near(got[0], host(y), NORM, "y")
    near(got[4], host(out), NORM, "out")
    near(got[5], host(n), NORM, "n")
    names = ["x", "r", "wa", "s", "wb", "rows", "z", "w", "q", "k", "v", "g", "beta", "h0"]
    for name, t in zip(names, got[8:]):
        if name in want:
            near(t.view(want[name].shape), host(want[name]), 16 * GRAD, name)    # (two norms' and the rule's, and dg's cancellation)
