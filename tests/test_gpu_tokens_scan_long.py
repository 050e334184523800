"""The selective scan on sequences of many tiles against the 64-bit definition: in one piece, where the loop over whole tiles runs,
and in chunks side by side, where every chunk starts from what those before it (backward: behind it) leave.  Which of the two
a plan takes is asserted from the kernels it names.
Chains as in test_gpu_tokens_scan: 4 L + N + 16, three times that for a gradient, and the terms of its sum."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import tokens as ot                        # noqa: E402
from token_helpers import DEV, TYPES, Gen, check, host     # noqa: E402


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


# B, L, D, N, groups, forward in chunks, backward in chunks
CASES = [(1, 400, 20, 16, 1, True, True), (1, 411, 90, 16, 1, True, True), (2, 333, 24, 5, 2, True, True), (1, 420, 300, 1, 1, True, True),
         (1, 390, 18, 64, 1, True, True), (1, 400, 33, 32, 1, True, True), (2, 350, 10, 8, 2, True, True), (1, 365, 30, 2, 1, True, True),
         (1, 352, 40, 13, 2, True, True), (2, 340, 12, 3, 1, True, True), (1, 400, 20, 33, 1, True, True), (1, 360, 260, 4, 2, True, True),
         (1, 200, 20, 16, 1, False, True), (1, 1300, 16, 16, 1, True, True), (1, 643, 128, 16, 64, True, True),
         (1, 660, 40, 5, 40, True, True), (1, 150, 256, 16, 256, False, False), (1, 261, 256, 5, 256, False, False),
         (1, 200, 256, 1, 256, False, False), (1, 177, 256, 32, 256, False, False), (1, 176, 256, 64, 256, False, False),
         (2, 190, 256, 8, 128, False, False), (1, 160, 256, 2, 256, False, False), (1, 240, 768, 3, 256, False, False)]


def _inputs(case, dtype, lens):
    B, L, D, N, G = case[:5]
    T = TYPES[dtype][0]
    g = Gen(sum(case[:5]))
    # steps of about 0.1 and decays down to 0.05: what a chunk starts from is still there hundreds of tokens on
    return dict(x=g.normal(B, L, D, dtype=T), dt=g.normal(B, L, D, dtype=T, mean=-2.0), A=-torch.exp(g.uniform(D, N, lo=-3.0, hi=2.0)),
                B=g.normal(B, L, G, N, dtype=T), C=g.normal(B, L, G, N, dtype=T), skip=g.normal(D), z=g.normal(B, L, D, dtype=T),
                dt_bias=g.normal(D, std=0.5), h0=g.normal(B, D, N, std=3.0), dy=g.normal(B, L, D, dtype=T), dh=g.normal(B, D, N, std=3.0),
                lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV))


def _run(mb, case, dtype, names, lens, softplus=True):
    B, L, D, N, G, forward, backward = case
    v = _inputs(case, dtype, lens)
    if not softplus:
        v["dt"] = v["dt"].abs() * 0.05
    extra = {k: v[k] for k in names if v[k] is not None}
    plan = mb.merit_plan_scan(TYPES[dtype][1], B, L, D, N, G, softplus)
    assert plan.kernel() == "merit_scan_tiles+merit_scan_tiles" if forward else plan.kernel() == "merit_scan_tiles"
    assert plan.kernel(mb.MERIT_PASS_BACKWARD).startswith("merit_scan_back_chunks+" if backward else "merit_scan_back+")
    five = (v["x"], v["dt"], v["A"], v["B"], v["C"])
    args, e = [host(t) for t in five], {k: (t.cpu().numpy() if k == "lens" else host(t)) for k, t in extra.items()}
    chain = 4 * L + N + 16

    y, h, states = mb.merit_scan(plan, *five, final=True, states=True, **extra)
    wy, wh, ws = ot.scan(*args, softplus=softplus, **e)
    check(y, wy, chain, "y")
    check(h, wh, chain, "h")
    h0 = e.get("h0", np.zeros_like(wh))
    for b in range(B):                                   # the states before every 16th token of the sequence
        n = L if lens is None else min(max(lens[b], 0), L)
        k = np.arange(-(-n // 16))
        if k.size:
            check(states[b, :k.size], np.where((k > 0)[:, None, None], ws[b, np.maximum(16 * k - 1, 0)], h0[b]), chain, "states")
    again, last = mb.merit_scan(plan, *five, final=True, **extra)        # (the kernel that keeps no states)
    assert torch.equal(again, y) and torch.equal(last, h)

    more = {k: t for k, t in extra.items() if k != "h0"}
    dh = v["dh"] if "h0" in extra else None
    got = mb.merit_scan_backward(plan, v["dy"], *five, states, dh_last=dh, dh0=True, **more)
    want = ot.scan_backward(host(v["dy"]), *args, dh_last=host(dh), softplus=softplus, **e)
    sums = {"dB": D // G, "dC": D // G, "dA": B * L, "dskip": B * L, "ddt_bias": B * L}
    for k, r in want.items():
        if k in ("dz", "dskip", "ddt_bias") and k[1:] not in extra:
            assert got[k] is None, k
        else:
            check(got[k], r, 3 * chain + sums.get(k, 0), k)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_whole_sequences(mb, case, dtype):
    _run(mb, case, dtype, ("skip", "z", "dt_bias"), None)
    _run(mb, case, dtype, ("skip", "h0"), None, softplus=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N, G", [(16, 1), (5, 1), (1, 1), (64, 1), (16, 4), (8, 2), (32, 1)])
def test_lengths_of_their_own(mb, N, G, dtype):
    """Sequences that end before the first token, in the first chunk, at and beside the ends of tiles (and so of chunks), in the
    last chunk, and not at all; states in and out, and their gradients."""
    ends = (400, 0, 1, 16, 37, 80, 96, 112, 160, 161, 200, 240, 320, 399, 384)
    for names in (("skip", "z", "dt_bias", "h0", "lens"), ("z", "lens")):
        _run(mb, (len(ends), 400, 12, N, G, True, True), dtype, names, ends)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("N", [16, 5, 2])
def test_lengths_in_one_piece(mb, N, dtype):
    ends = (300, 0, 128, 129, 143, 300, 260, 17)
    _run(mb, (len(ends), 300, 64, N, 32, False, False), dtype, ("skip", "z", "dt_bias", "h0", "lens"), ends)


def test_nothing_behind_an_end_is_read_in_chunks(mb):
    B, L, D, N = 4, 400, 20, 16
    ends = (400, 37, 160, 0)
    v = _inputs((B, L, D, N, 1), "f32", ends)
    plan = mb.merit_plan_scan(TYPES["f32"][1], B, L, D, N)
    d = {k: v[k].clone() for k in ("x", "dt", "B", "C", "z", "dy")}
    for b, n in enumerate(ends):
        for k, t in d.items():
            t[b, n:] = float("nan") if k in ("x", "B", "dy") else float("inf")
    kw = dict(skip=v["skip"], dt_bias=v["dt_bias"], lens=v["lens"])
    results = []
    for u in (v, {**v, **d}):
        y, h, st = mb.merit_scan(plan, u["x"], u["dt"], v["A"], u["B"], u["C"], z=u["z"], h0=v["h0"], final=True, states=True, **kw)
        g = mb.merit_scan_backward(plan, u["dy"], u["x"], u["dt"], v["A"], u["B"], u["C"], st, z=u["z"], dh_last=v["dh"], dh0=True, **kw)
        results.append([y, h, *g.values()])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_gradients_of_16_bit_tensors_against_differences(mb):
    """Differences of the fp32 kernel at inputs that binary16 holds, against the binary16 kernel's gradients there: next to the
    differences' own error (test_gpu_tokens_scan: 2 % of their norm) each rounding of a result, 2^-11 of it, is nothing."""
    B, L, D, N, G = 1, 6, 4, 3, 1
    T, code, _ = TYPES["f16"]
    g = Gen(3)
    v = dict(x=g.normal(B, L, D), dt=g.normal(B, L, D, mean=-2.0), A=-g.uniform(D, N, lo=0.1, hi=8.0), B=g.normal(B, L, G, N),
             C=g.normal(B, L, G, N), skip=g.normal(D), z=g.normal(B, L, D), dt_bias=g.normal(D, std=0.5), h0=g.normal(B, D, N),
             dy=g.normal(B, L, D), dh=g.normal(B, D, N))
    v = {k: t.to(T).float() for k, t in v.items()}
    tensors, names = ("x", "dt", "B", "C", "z", "dy"), ("skip", "z", "dt_bias", "h0")
    plan, half = mb.merit_plan_scan(TYPES["f32"][1], B, L, D, N, G), mb.merit_plan_scan(code, B, L, D, N, G)

    def total(**new):
        u = {**v, **new}
        y, h = mb.merit_scan(plan, u["x"], u["dt"], u["A"], u["B"], u["C"], final=True, **{k: u[k] for k in names})
        return float((y.double() * v["dy"].double()).sum() + (h.double() * v["dh"].double()).sum())

    u = {k: t.to(T) if k in tensors else t for k, t in v.items()}
    five = (u["x"], u["dt"], u["A"], u["B"], u["C"])
    _, states = mb.merit_scan(half, *five, states=True, **{k: u[k] for k in names})
    got = mb.merit_scan_backward(half, u["dy"], *five, states, skip=u["skip"], z=u["z"], dt_bias=u["dt_bias"], dh_last=u["dh"], dh0=True)
    step = 2.0 ** -6
    for k in ("x", "dt", "A", "B", "C", "skip", "z", "dt_bias", "h0"):
        t, num = v[k], torch.zeros(v[k].numel(), dtype=torch.float64)
        for i in range(t.numel()):
            up, down = t.clone(), t.clone()
            up.view(-1)[i] += step
            down.view(-1)[i] -= step
            num[i] = (total(**{k: up}) - total(**{k: down})) / (2 * step)
        assert got["d" + k].dtype == (T if k in tensors else torch.float32)
        d = (num - got["d" + k].double().cpu().view(-1)).norm() / num.norm()
        assert d < 0.02, (k, float(d))
