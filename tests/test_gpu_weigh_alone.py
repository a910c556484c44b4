"""What a sequence's rows pay does not depend on which other sequences a call has beside it."""
import pytest
import torch

from paper_2601_13143_b200 import fastav
from test_gpu_attend import Problem, _cu
from test_gpu_weigh import Weighing, _dev

pytestmark = pytest.mark.gpu


def _weights(p, w, sequences):
    """The pool after a call with these sequences alone."""
    pool, cu = w.weights.cuda(), _cu(p.rows).tolist()
    rows = torch.cat([torch.arange(cu[b], cu[b + 1]) for b in sequences])
    q, counts, lens = p.q[rows].cuda(), [p.rows[b] for b in sequences], [p.lens[b] for b in sequences]
    params = p.params(batch=len(sequences), total_q=len(rows), max_qlen=max(counts), max_kv_len=max(lens))
    fastav.fastav_cache_weigh(params, p.cache, pool, q, w.lse[rows].cuda(), _cu(counts).cuda(), p.tables[0][list(sequences)].contiguous().cuda(), _dev(lens),
                              device_status=p.status)
    assert int(p.status) == 0
    return pool.cpu()


@pytest.mark.parametrize("hq,hkv,dim,fmt,rows", [(16, 4, 128, "int8", 100), (8, 2, 64, "fp8", 260), (32, 8, 128, "int8", 73), (12, 4, 128, "fp8", 7)])
def test_equal_bits_alone_and_in_a_batch(hq, hkv, dim, fmt, rows):
    """Several row tiles (and one), and lengths that lay the edges of the blocks' runs anywhere: units are taken singly and in pairs."""
    lens = [900, 2000, 31, 1300, 128, 3000, 640, 257, 1025]
    p = Problem(hq, hkv, dim, fmt, 32, lens, [min(rows, n) for n in lens], seed=3)
    w = Weighing(p)
    together = _weights(p, w, range(len(lens)))
    some = _weights(p, w, (1, 3, 5))
    for b in range(len(lens)):
        if p.rows[b] * (hq // hkv) <= 16:
            continue                                     # the kernel for few rows takes it by itself
        to, slot, _ = w.at[b]
        alone = _weights(p, w, (b,))
        for pool in (together, some) if b in (1, 3, 5) else (together,):
            assert torch.equal(pool[to, :, slot], alone[to, :, slot]), b


@pytest.mark.parametrize("dim,fmt", [(64, "int8"), (128, "fp8")])
def test_equal_bits_alone_and_in_a_batch_for_few_rows(dim, fmt):
    """16 stacked rows beside 4, 8 and 12."""
    lens = [900, 31, 1300, 128, 3000]
    p = Problem(16, 4, dim, fmt, 16, lens, [1, 2, 4, 3, 2], seed=4)
    w = Weighing(p)
    together = _weights(p, w, range(len(lens)))
    for b in range(len(lens)):
        to, slot, _ = w.at[b]
        assert torch.equal(together[to, :, slot], _weights(p, w, (b,))[to, :, slot]), b
