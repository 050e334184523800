"""Plans whose passes need about as many threads as a launch holds (fewer than 2^32).  No GPU: the kernels that a plan names."""
import pytest

from paper_1911_03458_amd import binding as mb


def _launches(plan, which=mb.MERIT_PASS_FORWARD):
    return plan.kernel(which).split("+")


@pytest.mark.parametrize("B, G, launches", [
    ((1 << 20) - 1, 8, 1),                               # 2^23 - 8 workgroups of 512 threads
    (1 << 20, 8, 2),                                     # 2^32 threads
    (8192, 1024, 2),
    ((1 << 24) - 2, 1, 2),
    ((1 << 24) - 1, 1, 3),                               # the most workgroups that a plan has
])
def test_scan_over_many_short_sequences(B, G, launches):
    plan = mb.merit_plan_scan(mb.MERIT_BF16, B, 1, G, 1, G)
    assert _launches(plan) == ["merit_scan_tiles"] * launches
    assert _launches(plan, mb.MERIT_PASS_STEP) == ["merit_scan_token"]
    assert _launches(plan, mb.MERIT_PASS_BACKWARD)[0] == "merit_scan_back"
