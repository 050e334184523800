"""Plans of the gated delta rule and of the block's norms: what they refuse, what scratch memory and kernels they say.  No GPU."""
import ctypes

import pytest
import torch

from paper_1911_03458_amd import binding as mb
from paper_1911_03458_amd import mixers, tokens

INVALID, SHAPE, UNSUPPORTED = mb.MERIT_ERR_INVALID_ARG, mb.MERIT_ERR_SHAPE, mb.MERIT_ERR_UNSUPPORTED
INF, NAN = float("inf"), float("nan")


def _refused(status, f, *args, **kw):
    with pytest.raises(mb.MeritError) as e:
        f(*args, **kw)
    assert e.value.status == status, e.value


@pytest.mark.parametrize("args, status", [
    ((0, 1, 8, 2, 1, 16, 16), INVALID), ((7, 1, 8, 2, 1, 16, 16), INVALID), ((2, -1, 8, 2, 1, 16, 16), INVALID),
    ((2, 1, -8, 2, 1, 16, 16), INVALID), ((2, 1, 8, 0, 1, 16, 16), INVALID), ((2, 1, 8, 2, 0, 16, 16), INVALID),
    ((2, 1, 8, 2, 1, 0, 16), INVALID), ((2, 1, 8, 2, 1, 16, 0), INVALID), ((2, 1, 8, 3, 2, 16, 16), SHAPE),
    ((2, 1, 8, 1, 2, 16, 16), SHAPE), ((2, 1, 8, 2, 1, 129, 16), UNSUPPORTED), ((2, 1, 1 << 31, 2, 1, 16, 16), UNSUPPORTED),
    ((2, 1 << 31, 8, 2, 1, 16, 16), UNSUPPORTED), ((2, 1 << 24, 8, 2, 1, 16, 16), UNSUPPORTED),      # more workgroups than a launch holds
    ((2, 1, 8, 1 << 20, 1, 16, 64), UNSUPPORTED), ((2, 1 << 12, 1 << 20, 2, 1, 16, 16), UNSUPPORTED),
])
def test_delta_plans_refused(args, status):
    _refused(status, mb.merit_plan_delta_rule, *args)


def test_delta_scales_refused():
    for scale in (INF, NAN):
        _refused(INVALID, mb.merit_plan_delta_rule, 2, 1, 8, 2, 1, 16, 16, scale=scale)


@pytest.mark.parametrize("args, kw, status", [
    ((0, 1, 8, 16), {}, INVALID), ((1, 1, 8, 16), dict(stream=3), INVALID), ((2, 1, 8, 16), dict(stream=1), INVALID),
    ((2, -1, 8, 16), {}, INVALID), ((2, 1, -1, 16), {}, INVALID), ((2, 1, 8, 0), {}, INVALID), ((2, 1, 8, 16), dict(eps=-1e-6), INVALID),
    ((2, 1, 8, 16), dict(eps=NAN), INVALID), ((2, 1, 8, 16), dict(eps=INF), INVALID), ((2, 1, 8, 16), dict(act=4), INVALID),
    ((2, 1, 8, 16), dict(act=-1), INVALID), ((2, 1, 8, 16), dict(after=False, before=False), INVALID),
    ((2, 1, 8, 16385), {}, UNSUPPORTED), ((2, 1 << 20, 1 << 20, 16), {}, UNSUPPORTED), ((2, 1, 1 << 31, 16), {}, UNSUPPORTED),
])
def test_block_norm_plans_refused(args, kw, status):
    _refused(status, mb.merit_plan_block_norm, *args, **kw)


def test_the_sigmoid_is_a_gate_only():
    mb.merit_plan_block_norm(2, 1, 8, 16, act=mb.MERIT_ACT_SIGMOID)
    _refused(INVALID, mb.merit_plan_group_norm, 2, 1, 1, 16, 1, 1e-5, mb.MERIT_ACT_SIGMOID)
    _refused(INVALID, mb.merit_plan_causal_conv, 2, 1, 8, 16, 4, mb.MERIT_ACT_SIGMOID)


def test_null_arguments_and_other_plans():
    L = mb.lib()
    n, s = ctypes.c_int64(), ctypes.c_char_p()
    assert L.merit_plan_delta_rule(2, 1, 8, 2, 1, 16, 16, 1.0, 1, None) == mb.MERIT_ERR_NULL
    assert L.merit_plan_block_norm(2, 2, 1, 8, 16, 1e-6, 0, 0, 1, 1, None) == mb.MERIT_ERR_NULL
    delta, norm, scan = mb.merit_plan_delta_rule(2, 2, 3, 2, 1, 8, 8), mb.merit_plan_block_norm(2, 2, 3, 8), mb.merit_plan_scan(2, 2, 3, 8, 4)
    views = (tokens.merit_view * 24)()
    for name in mixers._ENTRIES:
        own, others = (delta, (norm, scan)) if "delta" in name else (norm, (delta, scan))
        f = getattr(L, name)
        assert f(None, ctypes.byref(views), None, 0, None) == mb.MERIT_ERR_NULL
        assert f(own.handle, None, None, 0, None) == mb.MERIT_ERR_NULL
        for other in others:
            assert f(other.handle, ctypes.byref(views), None, 0, None) == INVALID
        assert f(own.handle, ctypes.byref(views), None, 0, None) == mb.MERIT_ERR_NULL    # the first required operand
    for name in tokens._ENTRIES:
        assert getattr(L, name)(delta.handle, ctypes.byref(views), None, 0, None) == INVALID
    for plan, step in ((delta, mb.MERIT_OK), (norm, INVALID)):
        assert L.merit_token_plan_workspace(plan.handle, 0, None) == mb.MERIT_ERR_NULL
        assert L.merit_token_plan_workspace(plan.handle, 2, ctypes.byref(n)) == step and n.value == 0
        assert L.merit_token_plan_workspace(plan.handle, 3, ctypes.byref(n)) == INVALID
        assert L.merit_token_plan_kernel(plan.handle, 2, ctypes.byref(s)) == step


def _fill(n, dtype):
    """Views of host addresses that nothing reads: the calls below end before a launch."""
    v = (tokens.merit_view * n)()
    for i in range(n):
        v[i] = tokens.merit_view(4096, (ctypes.c_int64 * 2)(64, 64), dtype, 0)
    return v


def test_operands_refused():
    L = mb.lib()
    plan = mb.merit_plan_delta_rule(mb.MERIT_F16, 2, 70, 2, 1, 8, 8)
    call, need = (lambda w=None, b=0: L.merit_delta_rule(plan.handle, ctypes.byref(v), w, b, None)), plan.workspace(0)
    v = _fill(10, mb.MERIT_F16)
    for i in (3, 5, 8, 9):
        v[i].dtype = mb.MERIT_F32
    assert need > 0 and call(None, need) == mb.MERIT_ERR_NULL
    assert call(4100, need) == mb.MERIT_ERR_ALIGNMENT
    assert call(4096, need - 1) == INVALID
    for i, wrong in ((0, mb.MERIT_BF16), (3, mb.MERIT_F16), (4, mb.MERIT_BF16), (5, mb.MERIT_F16), (7, mb.MERIT_F32), (9, mb.MERIT_F16)):
        kept, v[i].dtype = v[i].dtype, wrong
        assert call(4096, need) == INVALID, i
        v[i].dtype = kept
    for i, at in ((0, 4097), (3, 4098), (4, 4097), (5, 4098), (6, 4098)):
        v[i].data = at
        assert call(4096, need) == mb.MERIT_ERR_ALIGNMENT, i
        v[i].data = 4096
    norm = mb.merit_plan_block_norm(mb.MERIT_F16, 2, 70, 8, stream=mb.MERIT_F32, before=False)
    v = _fill(14, mb.MERIT_F16)
    for i in (2, 8, 10, 11, 12, 13):
        v[i].dtype = mb.MERIT_F32
    assert L.merit_block_norm(norm.handle, ctypes.byref(v), None, 0, None) == INVALID     # a norm's weight without the norm
    v[2].dtype = mb.MERIT_F16                                                                # the stream has a type of its own
    v[6].data = v[7].data = v[9].data = None
    assert L.merit_block_norm(norm.handle, ctypes.byref(v), None, 0, None) == INVALID


def test_scratch_and_kernels():
    plan = mb.merit_plan_delta_rule(mb.MERIT_BF16, 2, 130, 4, 2, 64, 64)
    assert plan.workspace(1) > plan.workspace(0) > 0 and plan.workspace(2) == 0
    assert plan.kernel() == "merit_delta_prepare+merit_delta_chunks"
    few = mb.merit_plan_delta_rule(mb.MERIT_BF16, 1, 8191, 16, 16, 128, 128)
    assert few.kernel() == "merit_delta_prepare+merit_delta_chunks+merit_delta_join+merit_delta_chunks"
    chunks = 128 * 16 * 9728 * 4
    assert 0 < few.workspace(0) - chunks <= 16 * 4 * 128 * 128 * 2 * 16 and (few.workspace(0) - chunks) % (16 * 128 * 128 * 4) == 0
    for one in ((8, 2048, 16), (1, 64, 1), (1, 0, 1), (300, 4096, 1)):
        assert mb.merit_plan_delta_rule(mb.MERIT_F32, one[0], one[1], one[2], one[2], 128, 128).kernel().count("chunks") == 1
    assert plan.kernel(mb.MERIT_PASS_STEP) == "merit_delta_token"
    assert plan.kernel(mb.MERIT_PASS_BACKWARD) == "merit_delta_back_chunks+merit_delta_grads+merit_delta_sum_heads"
    assert mb.merit_plan_delta_rule(mb.MERIT_BF16, 2, 0, 4, 2, 64, 64).workspace(1) == 0
    norm = mb.merit_plan_block_norm(mb.MERIT_BF16, 2, 130, 64)
    assert norm.workspace(0) == 0 and norm.workspace(1) > 0
    assert norm.kernel() == "merit_block_norm_rows"
    assert norm.kernel(mb.MERIT_PASS_BACKWARD) == "merit_block_norm_rows_backward+merit_reduce_rows"


def test_empty_batches_are_no_work():
    L = mb.lib()
    v = (tokens.merit_view * 24)()
    delta = mb.merit_plan_delta_rule(2, 0, 3, 2, 1, 8, 8)
    for name in ("merit_delta_rule", "merit_delta_rule_backward", "merit_delta_rule_step"):
        assert getattr(L, name)(delta.handle, ctypes.byref(v), None, 0, None) == mb.MERIT_OK
    for B, n in ((0, 3), (3, 0)):
        norm = mb.merit_plan_block_norm(2, B, n, 8)
        for name in ("merit_block_norm", "merit_block_norm_backward"):
            assert getattr(L, name)(norm.handle, ctypes.byref(v), None, 0, None) == mb.MERIT_OK


def test_host_tensors_and_other_plans_refused():
    plan = mb.merit_plan_block_norm(mb.MERIT_F32, 1, 4, 8)
    with pytest.raises(TypeError, match="device tensor"):
        mb.merit_block_norm(plan, torch.zeros(1, 4, 8))
    with pytest.raises(mb.MeritError):
        mb.merit_delta_rule_step(plan, *[None] * 6)
    with pytest.raises(mb.MeritError):
        mb.merit_block_norm(mb.merit_plan_delta_rule(mb.MERIT_F32, 1, 4, 1, 1, 8, 8), torch.zeros(1, 4, 8))
    plan.destroy()
    with pytest.raises(ValueError, match="destroyed"):
        plan.handle
