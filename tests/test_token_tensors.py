"""What the binding refuses of the rotation's, the weighing's and the eviction's tensors, without a GPU: their addresses alone do not say how they are read."""
import pytest
import torch

from paper_2601_13143_b200 import build as fbuild
from paper_2601_13143_b200 import fastav


class _Stream:
    cuda_stream = 0


@pytest.fixture(scope="module", autouse=True)
def built():
    fbuild.build()
    fbuild.build_binding()


DIM = 64
BAD_NORMS = {
    "fp32": torch.ones(DIM),
    "fp32, as many bytes": torch.ones(DIM // 2),
    "fp16": torch.ones(DIM, dtype=torch.float16),
    "too short": torch.ones(DIM - 8, dtype=torch.bfloat16),
    "too long": torch.ones(2 * DIM, dtype=torch.bfloat16),
    "every other element": torch.ones(2 * DIM, dtype=torch.bfloat16)[::2],
}


@pytest.mark.parametrize("name", BAD_NORMS)
@pytest.mark.parametrize("side", ["q", "k"])
def test_norm_weights_that_are_no_row_of_bf16(name, side):
    x = torch.zeros(5, 2, DIM, dtype=torch.bfloat16)
    norms = [None, None]
    norms["qk".index(side)] = BAD_NORMS[name]
    params = fastav.make_rotate_params(q=x, k=x, v=x, q_out=x, k_out=x)
    cache, table = fastav.make_cache(3, 2, DIM, 32, device="cpu"), torch.zeros(1, 8, dtype=torch.int32)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="norm weights"):
        fastav.fastav_rotate(params, x, x, None, x, x, *norms, stream=_Stream)
    with pytest.raises(ValueError, match="norm weights"):
        fastav.fastav_rotate_write(params, cache, x, x, x, None, cu, table, None, x, *norms, stream=_Stream)


def test_norm_weights_that_are_right_get_to_the_library():
    """... which refuses the call for another reason (rotary_dim), ahead of the GPU; weights of a side that is not there are not looked at."""
    x, w = torch.zeros(5, 2, DIM, dtype=torch.bfloat16), torch.ones(DIM, dtype=torch.bfloat16)
    params = fastav.make_rotate_params(q=x, k=x, q_out=x, k_out=x)
    params.rotary_dim = 24
    for q, norm in ((x, w), (None, torch.ones(3))):
        with pytest.raises(fastav.FastavError):
            fastav.fastav_rotate(params, q, x, None, q, x, norm, w, stream=_Stream)
    with pytest.raises(fastav.FastavError):
        fastav.fastav_rotate(params, x, x, None, x, x, None, None, stream=_Stream)


POOL = (3, 2, 32)  # pages, KV heads, page tokens
BAD_WEIGHTS = {
    "int32": torch.zeros(POOL, dtype=torch.int32),
    "fp64, as many bytes": torch.zeros(3, 2, 16, dtype=torch.float64),
    "bf16": torch.zeros(POOL, dtype=torch.bfloat16),
    "a page too few": torch.zeros(2, 2, 32),
    "heads and tokens exchanged": torch.zeros(3, 32, 2).transpose(1, 2),
    "none": None,
}


@pytest.mark.parametrize("name", BAD_WEIGHTS)
def test_weights_that_are_no_pool_of_fp32(name):
    cache, table = fastav.make_cache(3, 2, DIM, 32, device="cpu"), torch.zeros(1, 3, dtype=torch.int32)
    assert tuple(cache.k_scale.shape) == POOL
    x, one = torch.zeros(5, 2, DIM, dtype=torch.bfloat16), torch.ones(1, dtype=torch.int32)
    attend = fastav.make_attend_params(batch=1, total_q=5, max_qlen=5, num_q_heads=2, max_kv_len=96, q=x, out=x, page_table=table)
    evict = fastav.make_evict_params(batch=1, max_kv_len=96, max_keep=10, page_table=table)
    with pytest.raises(ValueError, match="fp32 weights"):
        fastav.fastav_cache_weigh(attend, cache, BAD_WEIGHTS[name], x, torch.zeros(5, 2), torch.zeros(2, dtype=torch.int32), table, one, stream=_Stream)
    with pytest.raises(ValueError, match="fp32 weights"):
        fastav.fastav_cache_evict(evict, cache, BAD_WEIGHTS[name], table, one, one, one, torch.zeros(4096, dtype=torch.uint8), stream=_Stream)


def test_weights_that_are_right_get_to_the_library():
    cache, table, one = fastav.make_cache(3, 2, DIM, 32, device="cpu"), torch.zeros(1, 3, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    evict = fastav.make_evict_params(batch=1, max_kv_len=97, max_keep=10, page_table=table)      # more tokens than the table has places
    with pytest.raises(fastav.FastavError):
        fastav.fastav_cache_evict(evict, cache, torch.zeros_like(cache.k_scale), table, one, one, one, torch.zeros(4096, dtype=torch.uint8), stream=_Stream)


@pytest.mark.parametrize("bad", [256, 257, -256, -1, 4])
def test_an_axis_is_one_of_the_positions_rows(bad):
    """(Held as a byte, where 256 is 0.)"""
    x, pos = torch.zeros(5, 2, DIM, dtype=torch.bfloat16), torch.zeros(3, 5, dtype=torch.int32)
    with pytest.raises(ValueError, match="axis"):
        fastav.make_rotate_params(q=x, q_out=x, pos=pos, frequencies=[1.0] * 8, axis=[0, 1, 2, 0, 1, bad, 0, 0])
    p = fastav.make_rotate_params(q=x, q_out=x, pos=pos, frequencies=[1.0] * 8, axis=[0, 1, 2, 0, 1, 2, 0, 0, 7])   # (entries of pairs that are not turned do not count)
    assert list(p.axis[:9]) == [0, 1, 2, 0, 1, 2, 0, 0, 0]
