"""Host-side planning of fastav_attend, seen through its workspace sizes; no GPU."""
import ctypes

import pytest

from paper_2601_13143_b200 import build as fbuild
from paper_2601_13143_b200 import fastav
from test_cache_abi import _attend, _cache


@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fastav.library()


def _bytes(lib, **over):
    out = ctypes.c_size_t(0)
    assert lib.fastav_attend_workspace_bytes(ctypes.byref(_attend(**over)), ctypes.byref(_cache()), ctypes.byref(out)) == fastav.FASTAV_OK
    return out.value


@pytest.mark.parametrize("rows", [1, 2])
def test_rows_on_a_prefix_do_not_count_where_there_is_none(lib, rows):
    """Up to 8 stacked rows take tiles of 8, whatever the fields of prefixes hold in a call without one."""
    assert _bytes(lib, max_qlen=rows, max_prefix_q=12, max_prefix_len=1 << 20, prefix_table_stride=7) == _bytes(lib, max_qlen=rows)
