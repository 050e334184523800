"""Plans of the token operators: what they refuse, what scratch memory and kernels they say, views.  No GPU."""
import ctypes

import pytest
import torch

from paper_1911_03458_amd import binding as mb
from paper_1911_03458_amd import tokens

INVALID, SHAPE, UNSUPPORTED = mb.MERIT_ERR_INVALID_ARG, mb.MERIT_ERR_SHAPE, mb.MERIT_ERR_UNSUPPORTED


def _refused(status, f, *args):
    with pytest.raises(mb.MeritError) as e:
        f(*args)
    assert e.value.status == status, e.value


@pytest.mark.parametrize("args, status", [
    ((0, 1, 1, 8, 2, 1e-5, 0), INVALID),                 # bytes have no norm
    ((7, 1, 1, 8, 2, 1e-5, 0), INVALID),
    ((2, -1, 1, 8, 2, 1e-5, 0), INVALID),
    ((2, 1, -1, 8, 2, 1e-5, 0), INVALID),
    ((2, 1, 1, 0, 1, 1e-5, 0), INVALID),
    ((2, 1, 1, 8, 0, 1e-5, 0), INVALID),
    ((2, 1, 1, 8, 3, 1e-5, 0), SHAPE),
    ((2, 1, 1, 8, 2, -1e-5, 0), INVALID),
    ((2, 1, 1, 8, 2, float("nan"), 0), INVALID),
    ((2, 1, 1, 8, 2, float("inf"), 0), INVALID),
    ((2, 1, 1, 8, 2, 1e-5, 3), INVALID),
    ((2, 1, 1, 1 << 25, 1, 1e-5, 0), UNSUPPORTED),
    ((2, 1 << 31, 1, 8, 2, 1e-5, 0), UNSUPPORTED),
    ((2, 1 << 30, 2, 8, 2, 1e-5, 0), UNSUPPORTED),       # more workgroups than a launch holds
])
def test_group_norm_plans_refused(args, status):
    _refused(status, mb.merit_plan_group_norm, *args)


@pytest.mark.parametrize("args, status", [
    ((0, 1, 1, 8, 4, 0), INVALID), ((2, -1, 1, 8, 4, 0), INVALID), ((2, 1, -1, 8, 4, 0), INVALID),
    ((2, 1, 1, 0, 4, 0), INVALID), ((2, 1, 1, 8, 0, 0), INVALID), ((2, 1, 1, 8, 4, -1), INVALID),
    ((2, 1, 1, 8, 9, 0), UNSUPPORTED), ((2, 1, 1 << 31, 8, 4, 0), UNSUPPORTED), ((2, 1 << 30, 1, 64, 4, 0), UNSUPPORTED),
])
def test_causal_conv_plans_refused(args, status):
    _refused(status, mb.merit_plan_causal_conv, *args)


@pytest.mark.parametrize("args, status", [
    ((0, 1, 1, 8, 4), INVALID), ((2, -1, 1, 8, 4), INVALID), ((2, 1, -1, 8, 4), INVALID), ((2, 1, 1, 0, 4), INVALID),
    ((2, 1, 1, 8, 0), INVALID), ((2, 1, 1, 8, 4, 0), INVALID), ((2, 1, 1, 8, 4, 3), SHAPE),
    ((2, 1, 1, 8, 65), UNSUPPORTED), ((2, 1, 1 << 31, 8, 4), UNSUPPORTED), ((2, 1 << 24, 1 << 20, 64, 16), UNSUPPORTED),
])
def test_scan_plans_refused(args, status):
    _refused(status, mb.merit_plan_scan, *args)


def test_null_arguments():
    L = mb.lib()
    n, s = ctypes.c_int64(), ctypes.c_char_p()
    assert L.merit_plan_group_norm(2, 1, 1, 8, 2, 1e-5, 0, None) == mb.MERIT_ERR_NULL
    assert L.merit_plan_causal_conv(2, 1, 1, 8, 4, 0, None) == mb.MERIT_ERR_NULL
    assert L.merit_plan_scan(2, 1, 1, 8, 4, 1, 1, None) == mb.MERIT_ERR_NULL
    assert L.merit_token_plan_destroy(None) == mb.MERIT_ERR_NULL
    assert L.merit_token_plan_workspace(None, 0, ctypes.byref(n)) == mb.MERIT_ERR_NULL
    assert L.merit_token_plan_kernel(None, 0, ctypes.byref(s)) == mb.MERIT_ERR_NULL
    norm, conv, scan = (mb.merit_plan_group_norm(2, 2, 3, 8, 2), mb.merit_plan_causal_conv(2, 2, 3, 8, 4),
                        mb.merit_plan_scan(2, 2, 3, 8, 4))
    assert L.merit_token_plan_workspace(norm.handle, 0, None) == mb.MERIT_ERR_NULL
    assert L.merit_token_plan_workspace(norm.handle, 2, ctypes.byref(n)) == INVALID      # a norm has no step
    assert L.merit_token_plan_workspace(norm.handle, 3, ctypes.byref(n)) == INVALID
    views = (tokens.merit_view * 24)()
    for name in tokens._ENTRIES:
        own = norm if "norm" in name else conv if "conv" in name else scan
        other = conv if own is not conv else scan
        f = getattr(L, name)
        assert f(None, ctypes.byref(views), None, 0, None) == mb.MERIT_ERR_NULL
        assert f(own.handle, None, None, 0, None) == mb.MERIT_ERR_NULL
        assert f(other.handle, ctypes.byref(views), None, 0, None) == INVALID
        assert f(own.handle, ctypes.byref(views), None, 0, None) == mb.MERIT_ERR_NULL    # the first required operand


def _fill(n, dtype):
    """Views of host addresses that nothing reads: the calls below end before a launch."""
    v = (tokens.merit_view * n)()
    for i in range(n):
        v[i] = tokens.merit_view(4096, (ctypes.c_int64 * 2)(64, 64), dtype, 0)
    return v


def test_operands_refused():
    L = mb.lib()
    norm = mb.merit_plan_group_norm(mb.MERIT_F16, 2, 3, 8, 2)
    v = _fill(6, mb.MERIT_F16)
    for i in (4, 5):
        v[i].dtype = mb.MERIT_F32
    v[0].dtype = mb.MERIT_BF16                          # not the plan's type
    assert L.merit_group_norm(norm.handle, ctypes.byref(v), None, 0, None) == INVALID
    v[0].dtype = mb.MERIT_F16
    v[0].data = 4097
    assert L.merit_group_norm(norm.handle, ctypes.byref(v), None, 0, None) == mb.MERIT_ERR_ALIGNMENT
    v[0].data = 4096
    v[1].dtype = mb.MERIT_BF16                          # a parameter: the plan's type or fp32
    assert L.merit_group_norm(norm.handle, ctypes.byref(v), None, 0, None) == INVALID
    v[1].dtype, v[1].data = mb.MERIT_F32, 4098
    assert L.merit_group_norm(norm.handle, ctypes.byref(v), None, 0, None) == mb.MERIT_ERR_ALIGNMENT
    v[1].data = 4096
    v[4].dtype = mb.MERIT_F16                           # statistics are fp32
    assert L.merit_group_norm(norm.handle, ctypes.byref(v), None, 0, None) == INVALID
    v[4].dtype = mb.MERIT_F32
    need = norm.workspace(mb.MERIT_PASS_FORWARD)
    assert need > 0
    assert L.merit_group_norm(norm.handle, ctypes.byref(v), None, need, None) == mb.MERIT_ERR_NULL
    assert L.merit_group_norm(norm.handle, ctypes.byref(v), 4100, need, None) == mb.MERIT_ERR_ALIGNMENT
    assert L.merit_group_norm(norm.handle, ctypes.byref(v), 4096, 0, None) == INVALID


def test_empty_batches_are_no_work():
    L = mb.lib()
    v = (tokens.merit_view * 24)()
    for plan, name in ((mb.merit_plan_group_norm(2, 0, 3, 8, 2), "merit_group_norm"),
                       (mb.merit_plan_causal_conv(2, 0, 3, 8, 4), "merit_causal_conv"),
                       (mb.merit_plan_causal_conv(2, 0, 3, 8, 4), "merit_causal_conv_step"),
                       (mb.merit_plan_scan(2, 0, 3, 8, 4), "merit_scan"), (mb.merit_plan_scan(2, 0, 3, 8, 4), "merit_scan_step")):
        assert getattr(L, name)(plan.handle, ctypes.byref(v), None, 0, None) == mb.MERIT_OK


def test_kernels_named():
    assert mb.merit_plan_group_norm(1, 4096, 1, 1024, 16).kernel() == "merit_norm_rows"
    assert "merit_norm_rows_backward" in mb.merit_plan_group_norm(1, 4096, 1, 1024, 16).kernel(mb.MERIT_PASS_BACKWARD)
    assert mb.merit_plan_group_norm(1, 2, 4096, 64, 16).kernel() == "merit_norm_slab"
    assert mb.merit_plan_group_norm(1, 2, 40960, 64, 16).kernel() == "merit_norm_stats+merit_norm_apply"
    assert "merit_norm_sums" in mb.merit_plan_group_norm(1, 1, 4096, 64, 16).kernel(mb.MERIT_PASS_BACKWARD)
    assert mb.merit_plan_causal_conv(3, 2, 5, 64, 4).kernel(mb.MERIT_PASS_STEP) == "merit_cconv_step"
    assert mb.merit_plan_scan(3, 2, 5, 64, 16).kernel(mb.MERIT_PASS_STEP) == "merit_scan_token"
    with pytest.raises(mb.MeritError):
        mb.merit_plan_group_norm(1, 4, 1, 8, 2).kernel(mb.MERIT_PASS_STEP)


def test_host_tensors_and_other_plans_refused():
    plan = mb.merit_plan_causal_conv(mb.MERIT_F32, 1, 4, 8, 4)
    with pytest.raises(TypeError, match="device tensor"):
        mb.merit_causal_conv(plan, torch.zeros(1, 4, 8), torch.zeros(8, 4))
    with pytest.raises(TypeError, match="device tensor"):
        mb.merit_causal_conv(plan, None, torch.zeros(8, 4))
    with pytest.raises(mb.MeritError):
        mb.merit_group_norm(plan, torch.zeros(1, 4, 8))
    plan.destroy()
    with pytest.raises(ValueError, match="destroyed"):
        plan.handle


def test_views_are_as_the_header_has_them():
    assert ctypes.sizeof(tokens.merit_view) == 8 + 16 + 8
