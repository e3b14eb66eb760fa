"""The largest sizes that include/ef.h states: more rows than a call counts are a wrong argument, rows wider than it takes are a size."""
import pytest

import paper_1905_10936_amd as ef
from tests.test_layers_cpu import CALLS, call

WIDEST = 1 << 24


@pytest.mark.parametrize("name", CALLS)
def test_rows(name):
    assert call(name, rows=1 << 31) == ef.EF_ERR_ARG


@pytest.mark.parametrize("name,width,stride", [("ef_act_encode", "width", "x_stride"), ("ef_act_decode", "width", "y_stride"),
                                               ("ef_weight_grad", "width", None), ("ef_weight_grad", "out_width", "dz_stride")])
def test_widths(name, width, stride):
    wider = {width: WIDEST + 1}
    if stride:
        wider[stride] = WIDEST + 1
    assert call(name, rows=2, **wider) == ef.EF_ERR_SIZE
    assert call(name, rows=0, **wider) == ef.EF_ERR_SIZE
