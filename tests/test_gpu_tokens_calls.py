"""How the token operators are called: the same bits every time, through the native module and through ctypes, on other
streams, under stream capture; memory that a call hands back."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from token_helpers import DEV, TYPES, Gen     # noqa: E402


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


def _block(mb, dtype="bf16", B=2, L=70, D=64, N=16, seed=1):
    """Every entry point on one set of inputs: a function of the stream argument, which returns all results."""
    T, code, _ = TYPES[dtype]
    g = Gen(seed)
    x, z, dy, dt = (g.normal(B, L, D, dtype=T) for _ in range(4))
    w, b, A = g.normal(D, 4), g.normal(D), -g.uniform(D, N, lo=0.5, hi=4.0)
    Bm, Cm, h0 = g.normal(B, L, 1, N, dtype=T), g.normal(B, L, 1, N, dtype=T), g.normal(B, D, N)
    conv, scan = mb.merit_plan_causal_conv(code, B, L, D, 4, mb.MERIT_ACT_SILU), mb.merit_plan_scan(code, B, L, D, N)
    token, image = mb.merit_plan_group_norm(code, B * L, 1, D, 4), mb.merit_plan_group_norm(code, B, L, D, 4, 1e-5, mb.MERIT_ACT_SILU)

    def run(**kw):
        out = [mb.merit_causal_conv(conv, x, w, b, **kw)]
        out += mb.merit_causal_conv_backward(conv, dy, x, w, b, **kw)
        out += mb.merit_causal_conv_step(conv, x[:, :3], x[:, 3], w, b, **kw)
        y, h, st = mb.merit_scan(scan, x, dt, A, Bm, Cm, skip=b, z=z, h0=h0, final=True, states=True, **kw)
        out += [y, h, st]
        out += [t for t in mb.merit_scan_backward(scan, dy, x, dt, A, Bm, Cm, st, skip=b, z=z, **kw).values() if t is not None]
        out += mb.merit_scan_step(scan, h0, x[:, 0], dt[:, 0], A, Bm[:, 0], Cm[:, 0], **kw)
        for plan, v, d in ((token, x.view(B * L, 1, D), dy.view(B * L, 1, D)), (image, x, dy)):
            y, mean, rstd = mb.merit_group_norm(plan, v, b, b, stats=True, **kw)
            out += [y, mean, rstd]
            out += mb.merit_group_norm_backward(plan, d, v, mean, rstd, b, b, **kw)
        return out

    return run


def _same(a, b):
    return len(a) == len(b) and all(torch.equal(s, t) for s, t in zip(a, b))


def test_the_same_bits_every_time_and_by_either_way(mb, monkeypatch):
    run = _block(mb, B=3, L=200, D=200)
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
    run2 = _block(mb, B=3, L=200, D=200)                 # plans that have not met the module
    assert _same(run2(), first) and len(called) == 10


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


def test_under_capture(mb):
    """Recorded once, replayed between the program's own work: every replay as the eager call."""
    run = _block(mb)
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for i in range(4):
        for t in out:
            t.fill_(float(i))
        torch.randn(1000, device=DEV).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(out, want), i


def test_scratch_memory_is_handed_back(mb):
    run = _block(mb)
    run()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    out = run()
    del out
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == before


def test_wrapped_tensors_and_modes_go_the_general_way(mb):
    plan = mb.merit_plan_causal_conv(mb.MERIT_F32, 1, 8, 16, 4)
    x, w = torch.randn(1, 8, 16, device=DEV), torch.randn(16, 4, device=DEV)

    class Sub(torch.Tensor):
        pass

    y = mb.merit_causal_conv(plan, x, w)
    assert torch.equal(mb.merit_causal_conv(plan, x.as_subclass(Sub), w), y)
    assert torch.equal(mb.merit_causal_conv(plan, torch.nn.Parameter(x), torch.nn.Parameter(w)), y)
