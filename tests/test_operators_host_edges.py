"""Refusals of the operators around the attention that need no GPU, at the ends of what their documentation allows."""
import pytest

from paper_2405_10637_b200 import binding as lk

from test_operators_host import scaling, tables


def test_copy_limits_refuse():
    f = lk.lib().lckv_quant_set_copy_limits
    assert f(-2, 0) == lk.EINVAL and f(0, -2) == lk.EINVAL
    assert f(-1, -1) == lk.OK


@pytest.mark.parametrize("rot_dim,base,factor", [(4, 10000.0, 1e300), (4, 1e300, 1e5), (128, 1e300, 1e9)])
def test_rope_tables_refuse_a_base_that_overflows(rot_dim, base, factor):
    assert tables(rot_dim=rot_dim, s=scaling(kind=2, base=base, factor=factor)) == lk.EINVAL
