"""Calls of the rotation, the weighing and the eviction that are refused on the host, without a GPU: sizes whose products leave 32 bits."""
import ctypes

import pytest

from paper_2601_13143_b200 import build as fbuild
from paper_2601_13143_b200 import fastav
from test_cache_abi import FAKE, UNSUPPORTED, _cache
from test_token_abi import _rotate


@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fastav.library()


@pytest.mark.parametrize("heads", [(1 << 26) + 1, 1 << 28, 1 << 29, 1 << 30, 2 ** 31 - 1])
def test_more_heads_than_a_launch_counts(lib, heads):
    """Rows of a token times lanes of a row wrap to 0 at 2^30 heads, and a launch divides by what follows from them."""
    wide = dict(q_stride_tok=heads * 64, qo_stride_tok=heads * 64, num_q_heads=heads)
    assert lib.fastav_rotate(ctypes.byref(_rotate(**wide)), FAKE, None, FAKE, None, None, 2 * FAKE, None, None) == UNSUPPORTED
    assert lib.fastav_rotate(ctypes.byref(_rotate(**wide)), FAKE, FAKE, FAKE, None, None, 2 * FAKE, 2 * FAKE, None) == UNSUPPORTED
    k = dict(k_stride_tok=heads * 64, ko_stride_tok=heads * 64, num_kv_heads=heads)
    assert lib.fastav_rotate(ctypes.byref(_rotate(**k)), None, FAKE, FAKE, None, None, None, 2 * FAKE, None) == UNSUPPORTED
    c = _cache()
    assert lib.fastav_rotate_write(ctypes.byref(_rotate(**wide)), ctypes.byref(c), *[FAKE] * 8, 4, None, 2 * FAKE, None, None) == UNSUPPORTED
