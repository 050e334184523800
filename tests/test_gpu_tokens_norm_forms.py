"""Group norm at sizes that select each form of the kernels: a group a workgroup at 4 and 8 units a thread of 256 and of 1024
threads, 2, 4 and 8 channels a lane; chunks whose threads have many rows.  Chains as in test_gpu_tokens_norm."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import token_reference as ref                          # noqa: E402
from oracle import tokens as ot                        # noqa: E402
from token_helpers import ACTS, DEV, TYPES, Gen, host     # noqa: E402

CHAIN = 256


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1911_03458_amd import binding
    binding.lib()
    return binding


def _form(S, units):
    """Units a thread and threads that hold a group of S rows of `units` vectors (the rule of csrc/token_plan.cpp)."""
    return next((f for f in ((4, 256), (8, 256), (4, 1024), (8, 1024)) if S <= f[1] // units * f[0]), None)


# type, N, S, C, groups, channels a lane, (units a thread, threads)
SLAB = [("f16", 2, 900, 256, 32, 8, (4, 256)), ("f16", 2, 1999, 256, 32, 8, (8, 256)), ("bf16", 2, 3136, 256, 32, 8, (4, 1024)),
        ("f16", 1, 4999, 256, 32, 8, (8, 1024)), ("bf16", 2, 2000, 512, 32, 8, (4, 1024)), ("f16", 3, 333, 960, 16, 4, (8, 1024)),
        ("f16", 3, 333, 896, 16, 8, (4, 1024)),
        ("bf16", 4, 1003, 144, 36, 4, (4, 256)), ("f16", 4, 1900, 144, 36, 4, (8, 256)), ("bf16", 8, 4001, 32, 8, 4, (4, 1024)),
        ("f16", 8, 8100, 32, 8, 4, (8, 1024)), ("f32", 2, 3136, 128, 32, 4, (4, 1024)), ("f32", 2, 4100, 128, 32, 4, (8, 1024)),
        ("f32", 4, 700, 160, 8, 4, (4, 1024)), ("f32", 4, 1601, 160, 8, 4, (8, 1024)), ("f32", 2, 1001, 128, 32, 4, (4, 256)),
        ("f16", 2, 1021, 96, 48, 2, (4, 256)), ("bf16", 2, 2011, 96, 48, 2, (8, 256)), ("f16", 2, 4011, 96, 48, 2, (4, 1024)),
        ("bf16", 2, 7011, 96, 48, 2, (8, 1024)), ("f32", 4, 1201, 48, 8, 2, (4, 1024)), ("f32", 4, 2601, 48, 8, 2, (8, 1024)),
        ("f32", 8, 31, 1024, 4, 4, (8, 256)), ("f16", 3, 16, 8192, 16, 8, (4, 256))]
# type, N, S, C, groups: chunks, rows of whole batches a thread and more
CHUNKS = [("f16", 512, 3000, 64, 8), ("bf16", 40, 12544, 64, 8), ("f32", 64, 6000, 24, 2), ("bf16", 96, 9001, 15, 3), ("f16", 64, 4111, 36, 6),
          ("f32", 3, 20000, 64, 1), ("bf16", 2, 1000, 4160, 2), ("f32", 5, 777, 2056, 1)]


def _compare(mb, dtype, N, S, C, G, what, back):
    T, code, _ = TYPES[dtype]
    g = torch.Generator(device=DEV).manual_seed(N + S + C)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    x = (normal(N, S, C) * (0.3 + 1.7 * torch.rand(C, generator=g, device=DEV)) + normal(C)).to(T)
    dy, w, b = normal(N, S, C).to(T), 1.0 + 0.3 * normal(C), 0.5 * normal(C)
    kind = ("none", "silu")[(N + S) % 2]
    plan = mb.merit_plan_group_norm(code, N, S, C, G, 1e-5, ACTS[kind])
    assert plan.kernel() == what and plan.kernel(mb.MERIT_PASS_BACKWARD).startswith(back + "+")
    y, mean, rstd = mb.merit_group_norm(plan, x, w, b, stats=True)
    for t, r, k in zip((y, mean, rstd), ref.group_norm(x, G, w, b, 1e-5, kind), ("y", "mean", "rstd")):
        ref.near(t, r, CHAIN, k)
    got = mb.merit_group_norm_backward(plan, dy, x, mean, rstd, w, b)
    # (a parameter's gradient: N S terms by threads of at least 100 rows, those by hundreds)
    for t, r, k, chain in zip(got, ref.group_norm_backward(dy, x, G, w, b, 1e-5, kind), ("dx", "dw", "db"),
                              (4 * CHAIN, 4 * CHAIN + N * S // 16, 4 * CHAIN + N * S // 16)):
        ref.near(t, r, chain, k)
    assert torch.equal(mb.merit_group_norm_backward(plan, dy, x, mean, rstd, w, b, dx=dy)[0], got[0])
    assert torch.equal(mb.merit_group_norm(plan, x, w, b, y=x), y)


@pytest.mark.parametrize("dtype, N, S, C, G, vec, form", SLAB)
def test_a_group_a_workgroup(mb, dtype, N, S, C, G, vec, form):
    most = 4 if dtype == "f32" else 8
    assert (C // G) % vec == 0 and (vec == most or (C // G) % (2 * vec)) and _form(S, C // G // vec) == form
    _compare(mb, dtype, N, S, C, G, "merit_norm_slab", "merit_norm_slab_backward")


@pytest.mark.parametrize("dtype, N, S, C, G", CHUNKS)
def test_chunks(mb, dtype, N, S, C, G):
    _compare(mb, dtype, N, S, C, G, "merit_norm_stats+merit_norm_apply", "merit_norm_sums+merit_norm_apply_backward")


def test_the_reference(mb):
    """token_reference against the oracle."""
    g = Gen(41)
    x, dy, w, b = g.normal(3, 7, 12), g.normal(3, 7, 12), g.normal(12), g.normal(12)
    for kind in ("none", "silu", "relu"):
        for a, r in zip(ref.group_norm(x, 3, w, b, 1e-5, kind), ot.group_norm(host(x), 3, host(w), host(b), 1e-5, kind)):
            np.testing.assert_allclose(a.cpu().numpy(), r, rtol=1e-11, atol=1e-11)
        for a, r in zip(ref.group_norm_backward(dy, x, 3, w, b, 1e-5, kind),
                        ot.group_norm_backward(host(dy), host(x), 3, host(w), host(b), 1e-5, kind)):
            np.testing.assert_allclose(a.cpu().numpy(), r, rtol=1e-11, atol=1e-11)
