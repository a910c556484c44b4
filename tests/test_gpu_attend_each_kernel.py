"""What fastav_attend promises beyond plain inputs, for each of its kernels: rows that are not finite, pages outside the pool, host bounds, pools beyond 2^32
bytes, peaked weights, strides.  Tolerances as derived in test_gpu_attend.py."""
import math

import pytest
import torch

from attend_shapes import GROUP, ROWS, place
from paper_2601_13143_b200 import fastav
from test_gpu_attend import Problem

pytestmark = pytest.mark.gpu
SHAPE = dict(hq=2 * GROUP, hkv=2, dim=128)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("rows", ROWS[1:] + [4])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("what", ["k", "v"])
def test_rows_that_are_not_finite_reach_those_that_see_them_only(what, bad, rows, fmt):
    """A key of one KV head that the last two query rows see, written by fastav_cache_write; the rest as if it were not there."""
    n = 100
    p = Problem(fmt=fmt, page=64, lens=[n], rows=[rows], seed=12, **SHAPE)
    gen = torch.Generator().manual_seed(13)
    x = {name: torch.randn(n, 2, 128, generator=gen).to(torch.bfloat16) for name in "kv"}
    place(p, 0, k=x["k"], v=x["v"])
    at, head = n - 2, 1
    x[what][at, head, 77] = bad
    last = {name: t[at:at + 1].cuda() for name, t in x.items()}
    one = torch.tensor([0, 1], dtype=torch.int32).cuda()
    params = fastav.make_params(batch=1, total_tokens=1, max_seqlen=1, total_q=0, max_qlen=0, total_keep=0, max_keep=0, num_q_heads=2, num_kv_heads=2, head_dim=128,
                                hidden=0, k=last["k"], v=last["v"])
    fastav.fastav_cache_write(params, p.cache, last["k"], last["v"], one, None, None, p.tables[0].cuda(), torch.tensor([at], dtype=torch.int32).cuda())
    p.run()
    out, lse = p.out.cpu().float().clone(), p.lse.cpu().clone()
    seeing, heads = slice(rows - 2, rows), slice(head * GROUP, (head + 1) * GROUP)
    assert bool(torch.isnan(out[seeing, heads]).all())
    assert what == "v" or bool(torch.isnan(lse[seeing, heads]).all())
    # everything else is what it is without that row's bad element: the rows before do not see it, the other head's are finite
    place(p, 0, k=torch.where(torch.isfinite(x["k"]), x["k"], 0), v=torch.where(torch.isfinite(x["v"]), x["v"], 0))
    p.run()
    p.check()
    same = torch.ones(rows, 2 * GROUP, dtype=torch.bool)
    same[seeing, heads] = False
    assert torch.equal(out[same], p.out.cpu().float()[same]) and torch.equal(lse[same], p.lse.cpu()[same])


@pytest.mark.parametrize("rows", ROWS)
def test_a_query_row_that_is_not_a_number_stays_alone(rows):
    p = Problem(fmt="int8", page=64, lens=[300, 200], rows=[rows, rows], seed=14, **SHAPE)
    p.run()
    want = p.out.clone()
    p.qd[rows, 3, 7] = math.nan     # the first row of the second sequence, one head
    p.run()
    hit = torch.zeros(p.total, p.hq, dtype=torch.bool, device="cuda")
    hit[rows, 3] = True
    assert bool(torch.isnan(p.out[hit]).all()) and torch.equal(p.out[~hit], want[~hit])


@pytest.mark.parametrize("page_id", [1 << 30, -1, -2 ** 31])
@pytest.mark.parametrize("rows", ROWS)
def test_a_page_outside_the_pool_is_reported_and_harms_its_sequence_only(rows, page_id):
    p = Problem(fmt="int8", page=64, lens=[200, 190, 70], rows=[rows, rows, rows], seed=11, **SHAPE)
    p.tables[0][1, 1] = page_id
    p.run()
    p.check(fastav.FASTAV_DEV_BAD_INDEX, skip=(1,))


@pytest.mark.parametrize("rows", ROWS)
def test_host_bounds_may_be_larger_and_too_small_ones_are_reported(rows):
    p = Problem(fmt="int8", page=128, lens=[200, 90], rows=[rows, max(1, rows // 2)], seed=10, **SHAPE)
    p.run(p.params(max_qlen=min(p.total, rows + 1), max_kv_len=100000))
    p.check()
    p.run(p.params(max_kv_len=100))
    assert int(p.status) == fastav.FASTAV_DEV_SHAPE_MISMATCH


@pytest.mark.parametrize("rows", ROWS)
def test_more_rows_than_the_host_said_are_reported(rows):
    p = Problem(fmt="int8", page=128, lens=[200, 90], rows=[rows + 1, 1], seed=10, **SHAPE)
    p.run(p.params(max_qlen=rows))
    assert int(p.status) == fastav.FASTAV_DEV_SHAPE_MISMATCH


@pytest.mark.parametrize("spread", [0.0, 30.0])
@pytest.mark.parametrize("rows", ROWS)
def test_flat_and_peaked_weights(rows, spread):
    p = Problem(fmt="int8", page=64, lens=[1000, 300], rows=[rows, max(1, rows // 2)], spread=spread, seed=3, **SHAPE)
    p.run()
    p.check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim,fmt", [(64, "fp8"), (128, "int8")])
@pytest.mark.parametrize("rows", ROWS)
def test_mask_strides_and_scale(rows, dim, fmt, causal):
    p = Problem(2 * GROUP, 2, dim, fmt, 32, [40, 100, 7], [rows, 1, rows], causal=causal, strided=True, scale=0.3, seed=5)
    p.run()
    p.check()
    whole = p.out.as_strided((p.total, p.hq + 2, p.dim + 16), (p.out.stride(0), p.out.stride(1), 1), 0)
    untouched = torch.ones_like(whole, dtype=torch.bool)
    untouched[:, 1:p.hq + 1, 8:p.dim + 8] = False
    assert bool((whole[untouched] == 7).all())


@pytest.mark.parametrize("rows", ROWS)
def test_strided_rows_on_a_shared_prefix(rows):
    """Both levels' parts joined into a strided output, without causal mask."""
    p = Problem(2 * GROUP, 2, 128, "fp8", 32, [40, 9, 70], [rows, 1, rows], causal=False, strided=True, prefix_lens=[400], groups=[0, 2], seed=6)
    p.run()
    p.check()


@pytest.mark.parametrize("rows", ROWS[1:])
def test_offsets_beyond_32_bits(rows):
    hkv, dim, page = 8, 128, 256
    pages = (5 << 30) // (hkv * dim * page)
    cache = fastav.make_cache(pages, hkv, dim, page)
    p = Problem(hkv * GROUP, hkv, dim, "int8", page, [600], [rows], seed=13)
    table = torch.tensor([[pages - 1, 3, pages - 2, 0]], dtype=torch.int32)
    for i in range(3):
        for name in ("k", "v", "k_scale", "v_scale"):
            getattr(cache, name)[int(table[0, i])] = getattr(p.cache, name)[int(p.tables[0][0, i])]
    p.cache, p.tables[0] = cache, table
    p.run()
    p.check()
