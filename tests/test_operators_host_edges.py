"""Refusals of the operators around the attention that need no GPU, at the ends of what their documentation allows."""
from paper_2405_10637_b200 import binding as lk


def test_copy_limits_refuse():
    f = lk.lib().lckv_quant_set_copy_limits
    assert f(-2, 0) == lk.EINVAL and f(0, -2) == lk.EINVAL
    assert f(-1, -1) == lk.OK
