"""More of what the operators refuse before anything is launched, without a GPU."""
import ctypes as C

import pytest

from test_operator_refusals import attention, lib  # noqa: F401  (fixture)
from paper_2609_09800_b200 import hbf


@pytest.mark.parametrize("kw", [dict(out_row_stride=0), dict(out_head_stride=0)])
def test_attention_s_rows_on_top_of_each_other(lib, kw):  # noqa: F811
    assert lib.hbf_prefix_attention(C.byref(attention(**kw)), 256, 1 << 30, None) == hbf.E_INVAL
