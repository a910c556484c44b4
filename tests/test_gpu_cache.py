"""fastav_cache_write and fastav_cache_read against the definitions in 64 bits: codes, scales and values have to be equal."""
import math

import pytest
import torch

import cache_reference as ref
from paper_2601_13143_b200 import fastav

pytestmark = pytest.mark.gpu

FORMATS = {"int8": (fastav.FASTAV_CACHE_INT8, torch.int8), "fp8": (fastav.FASTAV_CACHE_FP8, torch.float8_e4m3fn)}
POISON = 0x55


def _cu(counts):
    return torch.tensor([0] + counts, dtype=torch.int64).cumsum(0).to(torch.int32)


def _cache(pages, heads, dim, page, fmt):
    cache = fastav.make_cache(pages, heads, dim, page, FORMATS[fmt][0])
    cache.k.view(torch.int8).fill_(POISON)
    cache.v.view(torch.int8).fill_(POISON)
    cache.k_scale.fill_(-3.0)
    cache.v_scale.fill_(-5.0)
    return cache


def _tables(gen, tokens, page, spare=2):
    need = [-(-n // page) for n in tokens]
    table = torch.full((len(tokens), max(need + [1]) + 1), -7, dtype=torch.int32)
    ids = torch.randperm(sum(need) + spare, generator=gen).to(torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = ids[at:at + m]
        at += m
    return table, sum(need) + spare


def _values(gen, n, heads, dim):
    """Rows of very different sizes, of few values, with ties, zeros, subnormal and huge ones."""
    x = torch.randn(n, heads, dim, generator=gen) * torch.exp2(torch.randint(-20, 20, (n, heads, 1), generator=gen).float())
    if n > 4:
        x[0] = 0
        x[1] = torch.randint(-127, 128, (heads, dim), generator=gen).float() / 2   # halves of codes: ties where 127 / 2 is the largest
        x[1, :, 0] = 63.5
        x[2] = x[2].sign() * 2.0 ** -133
        x[3] *= 2.0 ** 100
        x[4] = torch.randint(-16, 17, (heads, dim), generator=gen).float() * 28     # ties of e4m3 where 448 is the largest
        x[4, :, 1] = 448
    return x.to(torch.bfloat16)


def _make(lens, counts, start, heads, dim, page, fmt, packed, seed):
    gen = torch.Generator().manual_seed(seed)
    total = sum(lens)
    k, v = _values(gen, total, heads, dim), _values(gen, total, heads, dim)
    keep = None
    if counts is not None:
        keep = [torch.randperm(n, generator=gen)[:c].sort().values for n, c in zip(lens, counts)]
    table, pages = _tables(gen, [s + c for s, c in zip(start, counts or lens)], page)
    whole = torch.full((total, 3 * heads + 1, dim), 9.0, dtype=torch.bfloat16)
    whole[:, 1:1 + heads], whole[:, 1 + 2 * heads:] = k, v
    whole = whole.cuda()
    kd, vd = (whole[:, 1:1 + heads], whole[:, 1 + 2 * heads:]) if packed else (k.cuda(), v.cuda())
    return k, v, kd, vd, keep, table, pages


def _params(lens, counts, heads, dim, flags=0, **more):
    return fastav.make_params(batch=len(lens), total_tokens=sum(lens), max_seqlen=max(lens), total_q=0, max_qlen=0, total_keep=sum(counts or [0]),
                              max_keep=max(counts or [0]), num_q_heads=heads, num_kv_heads=heads, head_dim=dim, hidden=0, flags=flags, **more)


def _expect_pool(cache, table, page, rows, code):
    """The pools after rows = [(sequence, first token, x_k, x_v)] were written."""
    pools = [cache.k.view(torch.int8).cpu().clone(), cache.v.view(torch.int8).cpu().clone()]
    scales = [cache.k_scale.cpu().clone(), cache.v_scale.cpu().clone()]
    for b, first, xk, xv in rows:
        at = first + torch.arange(len(xk))
        for pool, scale, x in zip(pools, scales, (xk, xv)):
            c, s = ref.quantise(x, code)
            to = table[b].long()[at // page]
            pool[to, :, at % page] = c.to(torch.float32).to(code).view(torch.int8)
            scale[to, :, at % page] = s
    return pools, scales


def _same(cache, pools, scales):
    for got, want in zip((cache.k, cache.v), pools):
        got, want = got.view(torch.int8).cpu(), want
        if cache.k.dtype != torch.int8:  # -0 and 0 are one value
            got, want = (torch.where((x & 0x7F) == 0, torch.zeros_like(x), x) for x in (got, want))
        assert torch.equal(got, want)
    for got, want in zip((cache.k_scale, cache.v_scale), scales):
        assert torch.equal(got.cpu().nan_to_num(-99.0), want.nan_to_num(-99.0))


CASES = [  # lengths, kept, first token, KV heads, dim, page, packed, global indices
    ([1], None, [0], 1, 64, 16, False, False),
    ([1, 1, 1, 1, 1], None, [0, 15, 16, 700, 31], 4, 128, 16, True, False),
    ([0, 33, 0, 1, 257], None, [0, 0, 5, 63, 64], 2, 128, 64, False, False),
    ([300, 5, 64], [100, 5, 0], [7, 0, 0], 8, 64, 256, True, False),
    ([300, 5, 64], [100, 0, 33], [0, 0, 127], 3, 128, 128, True, True),
    ([2000, 3000], [1500, 999], [1, 2], 5, 128, 32, False, False),
    ([40000], None, [0], 2, 64, 64, False, False),
]


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_written_codes_scales_and_read_values(case, fmt):
    lens, counts, start, heads, dim, page, packed, global_idx = CASES[case]
    code = FORMATS[fmt][1]
    k, v, kd, vd, keep, table, pages = _make(lens, counts, start, heads, dim, page, fmt, packed, 100 + case)
    cache = _cache(pages, heads, dim, page, fmt)
    cu = _cu(lens).tolist()
    rows = []
    for b in range(len(lens)):
        src = cu[b] + (keep[b] if keep else torch.arange(lens[b]))
        rows.append((b, start[b], k[src], v[src]))
    pools, scales = _expect_pool(cache, table, page, rows, code)
    idx = None
    if keep:
        idx = torch.cat([kb + (cu[b] if global_idx else 0) for b, kb in enumerate(keep)]).to(torch.int32).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    params = _params(lens, counts, heads, dim, fastav.FASTAV_KEEP_IDX_GLOBAL if global_idx else 0, k=kd, v=vd)
    tabled, startd = table.cuda(), torch.tensor(start, dtype=torch.int32).cuda()
    fastav.fastav_cache_write(params, cache, kd, vd, _cu(lens).cuda(), idx, _cu(counts).cuda() if counts else None, tabled,
                              startd if any(start) else None, status)
    assert int(status) == 0
    _same(cache, pools, scales)

    moved = counts or lens
    out = torch.full((sum(moved), 2 * heads + 1, dim), 3.0, dtype=torch.bfloat16, device="cuda")
    ko, vo = out[:, :heads], out[:, heads + 1:]
    fastav.fastav_cache_read(_params(moved, None, heads, dim, k_out=ko, v_out=vo), cache, tabled, startd, _cu(moved).cuda(), ko, vo, status)
    assert int(status) == 0 and bool((out[:, heads] == 3).all())
    for got, pool, scale in ((ko, pools[0], scales[0]), (vo, pools[1], scales[1])):
        at = [(table[b].long()[t // page], t % page) for b, n in enumerate(moved) for t in [start[b] + torch.arange(n)]]
        to, slot = torch.cat([a for a, _ in at]), torch.cat([s for _, s in at])
        want = (pool[to, :, slot].view(code).float() * scale[to, :, slot][..., None]).to(torch.bfloat16)
        assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_row_that_is_not_finite_reads_back_as_nan_and_its_neighbours_do_not(fmt, bad):
    x = torch.randn(20, 2, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    x[7, 1, 100] = bad
    cache = _cache(2, 2, 128, 16, fmt)
    table = torch.tensor([[1, 0]], dtype=torch.int32).cuda()
    xd, y = x.cuda(), torch.empty_like(x).cuda()
    cu = _cu([20]).cuda()
    fastav.fastav_cache_write(_params([20], None, 2, 128, k=xd, v=xd), cache, xd, xd, cu, None, None, table)
    fastav.fastav_cache_read(_params([20], None, 2, 128, k_out=y, v_out=y), cache, table, None, cu, torch.empty_like(y), y)
    nan = torch.isnan(y.cpu())
    assert bool(nan[7, 1].all()) and int(nan.sum()) == 128
    assert not torch.isnan(cache.v.view(torch.float8_e4m3fn if fmt == "fp8" else torch.int8).float()).any()


def test_rows_without_a_place_are_left_out_and_reported():
    heads, dim, page = 2, 64, 16
    x = torch.randn(40, heads, dim).to(torch.bfloat16).cuda()
    table = torch.tensor([[0, 99], [1, -1]], dtype=torch.int32).cuda()
    cu, status = _cu([20, 20]).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = _cache(3, heads, dim, page, "int8")
    params = _params([20, 20], None, heads, dim, k=x, v=x)
    fastav.fastav_cache_write(params, cache, x, x, cu, None, None, table, None, status)
    assert int(status) == fastav.FASTAV_DEV_BAD_INDEX
    assert bool((cache.k[2] == POISON).all()) and not bool((cache.k[:2] == POISON).all(-1).any())
    y = torch.full_like(x, 3.0)
    status.zero_()
    fastav.fastav_cache_read(_params([20, 20], None, heads, dim, k_out=y, v_out=y), cache, table, None, cu, y, y, status)
    assert int(status) == fastav.FASTAV_DEV_BAD_INDEX
    assert bool((y[16:20] == 3).all()) and bool((y[36:] == 3).all()) and not bool((y[:16] == 3).all(-1).any())
    # behind the table's end, and before the sequence's begin
    for start in ([20, 0], [-1, 0], [2 ** 31 - 1, 0]):
        status.zero_()
        table2 = torch.tensor([[0, 1], [1, 2]], dtype=torch.int32).cuda()
        fastav.fastav_cache_write(params, cache, x, x, cu, None, None, table2, torch.tensor(start, dtype=torch.int32).cuda(), status)
        assert int(status) == fastav.FASTAV_DEV_SHAPE_MISMATCH
    # a survivor outside its sequence; more survivors than the host said
    status.zero_()
    idx = torch.tensor([0, 19, 20, 5], dtype=torch.int32).cuda()
    fastav.fastav_cache_write(_params([20, 20], [2, 2], heads, dim, k=x, v=x), cache, x, x, cu, idx, _cu([2, 2]).cuda(), table, None, status)
    assert int(status) == fastav.FASTAV_DEV_BAD_INDEX
    status.zero_()
    fastav.fastav_cache_write(_params([20, 20], [1, 2], heads, dim, k=x, v=x), cache, x, x, cu, idx, _cu([2, 2]).cuda(), table, None, status)
    assert int(status) & fastav.FASTAV_DEV_SHAPE_MISMATCH


def test_offsets_beyond_32_bits():
    """A pool whose last rows lie more than 2^32 bytes in."""
    heads, dim, page = 8, 128, 256
    pages = (5 << 30) // (heads * dim * page)
    cache = fastav.make_cache(pages, heads, dim, page)
    x = torch.randn(300, heads, dim, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32).cuda()
    xd, y, z = x.cuda(), torch.empty_like(x).cuda(), torch.empty_like(x).cuda()
    cu = _cu([300]).cuda()
    fastav.fastav_cache_write(_params([300], None, heads, dim, k=xd, v=xd), cache, xd, xd, cu, None, None, table)
    fastav.fastav_cache_read(_params([300], None, heads, dim, k_out=y, v_out=z), cache, table, None, cu, y, z)
    codes, scale = ref.quantise(x, torch.int8)
    want = (codes.float() * scale[..., None]).to(torch.bfloat16)
    assert torch.equal(y.cpu(), want) and torch.equal(z.cpu(), want)


def test_writes_what_earlier_work_on_the_stream_leaves():
    """Indices and rows made by kernels that run right before, on a stream of the caller's."""
    heads, dim, page, n = 4, 128, 64, 3000
    side = torch.cuda.Stream()
    x = torch.randn(n, heads, dim, device="cuda").to(torch.bfloat16)
    table = torch.arange(64, dtype=torch.int32, device="cuda")[None]
    cache = _cache(64, heads, dim, page, "int8")
    cu = _cu([n]).cuda()
    y = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for i in range(5):
            moved, flipped = x + i, table.flip(1) if i % 2 else table.clone()
            fastav.fastav_cache_write(_params([n], None, heads, dim, k=moved, v=moved), cache, moved, moved, cu, None, None, flipped)
            fastav.fastav_cache_read(_params([n], None, heads, dim, k_out=y, v_out=y), cache, flipped, None, cu, torch.empty_like(y), y)
            got = y.clone()
            side.synchronize()
            codes, scale = ref.quantise(moved.cpu(), torch.int8)
            assert torch.equal(got.cpu(), (codes.float() * scale[..., None]).to(torch.bfloat16))
