"""fastav_cache_weigh against the definition in 64 bits.

Tolerances.  A logit is a sum of exact products in fp32: head_dim / 16 steps of the matrix unit, each off by at most 2^-22 of the sum of magnitudes B, and
three products; it and the log-sum-exp are rounded in base 2 (2^-23 of either, and of their difference); the exponential is good to 2^-21.  So a row's part p of a weight is off by at most
    p (2^-22 (head_dim / 16 + 4) + 2^-20) (B + |lse| + 1)
and sums of R G parts by 2^-24 of themselves for each addition (a lane's few, then two across lanes; many rows: R G at most).  Parts below 2^-126 are
taken as 0 (the exponential leaves fp32's normal range there): each is off by less than 2^-126."""
import math

import pytest
import torch

import token_reference as ref
from paper_2601_13143_b200 import fastav
from test_gpu_attend import Problem, _cu

pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


class Weighing:
    """A problem of the attention's tests, weights in its places and hostile ones elsewhere, and log-sum-exps near the rows' own."""

    def __init__(self, p, decay=1.0, fresh=None, lse=None, seed=3):
        self.p, self.decay, self.fresh = p, decay, fresh
        gen = torch.Generator().manual_seed(seed)
        self.weights = torch.full(p.cache.k_scale.shape, math.nan)
        self.at = []
        for b, n in enumerate(p.lens):
            t = torch.arange(n)
            to, slot = p.tables[0][b].long()[t // p.page], t % p.page
            w = torch.rand(n, p.hkv, generator=gen) * 3
            if fresh is not None:
                w[max(0, min(n, fresh[b])):] = math.nan        # never read
            self.weights[to, :, slot] = w if decay else torch.full_like(w, math.nan)
            self.at.append((to, slot, w))
        scale = p.scale if p.scale > 0 else 1 / math.sqrt(p.dim)
        if lse is None:
            lse = torch.zeros(p.total, p.hq)
            cu = _cu(p.rows).tolist()
            for b, n in enumerate(p.lens):
                for r, sees in enumerate(p.sees(b)):
                    if sees <= 0 or n == 0:
                        lse[cu[b] + r] = -math.inf
                        continue
                    k = p.tokens[b][0][:sees].repeat_interleave(p.hq // p.hkv, 1)
                    lse[cu[b] + r] = torch.logsumexp(torch.einsum("nhd,hd->hn", k, p.q[cu[b] + r].double()) * scale, 1).float()
        self.lse, self.scale = lse, scale
        self.on_gpu = self.weights.cuda()

    def run(self, params=None, stream=None, status=None, **over):
        p = self.p
        fresh = None if self.fresh is None else _dev(self.fresh)
        a = dict(q=p.qd, lse=self.lse.cuda(), cu_qlens=_cu(p.rows).cuda(), page_table=p.tables[0].cuda(), kv_lens=_dev(p.lens), weighed_lens_opt=fresh)
        a.update(over)
        fastav.fastav_cache_weigh(params or p.params(), p.cache, self.on_gpu, decay=self.decay, device_status=p.status if status is None else status, stream=stream, **a)
        torch.cuda.synchronize()

    def check(self, status=0, skip=()):
        p, got = self.p, self.on_gpu.cpu()
        assert int(p.status) == status
        same = torch.ones(got.shape, dtype=torch.bool)
        cu = _cu(p.rows).tolist()
        for b, n in enumerate(p.lens):
            to, slot, w = self.at[b]
            same[to, :, slot] = False
            if b in skip or n == 0:
                continue
            fresh = n if self.fresh is None else max(0, min(n, self.fresh[b]))
            rows = slice(cu[b], cu[b + 1])
            want, size = ref.weigh(w, self.decay, fresh, p.q[rows], p.tokens[b][0], self.lse[rows], p.sees(b), self.scale)
            assert torch.isfinite(want).all()
            excess = (got[to, :, slot].double() - want).abs() - (size * (2.0 ** -22 * (p.dim / 16 + 4) + 2.0 ** -20) + 2.0 ** -24 * (4 + p.rows[b] * p.hq // p.hkv) * want + p.rows[b] * p.hq // p.hkv * 2.0 ** -126)
            assert float(excess.max()) <= 0, (b, float(excess.max()))
        assert torch.equal(got[same].nan_to_num(-1.0), self.weights[same].nan_to_num(-1.0))  # places of no sequence


CASES = {
    # hq, hkv, dim, page, lens, rows
    "one_key": (8, 2, 64, 16, [1], [1]),
    "lengths_around_a_unit": (28, 4, 128, 16, [31, 32, 33, 1, 64, 65, 17, 15, 16, 127, 128, 129], [1] * 12),
    "no_keys_and_no_rows": (8, 2, 128, 64, [0, 5, 0, 40], [1, 0, 0, 2]),
    "more_rows_than_keys": (8, 2, 128, 32, [3, 1, 0], [7, 4, 3]),
    "many_short": (32, 8, 128, 16, [7 + 13 * i % 61 for i in range(150)], [1] * 150),
    "one_head_long": (1, 1, 128, 64, [9001], [1]),
    "group_of_16": (32, 2, 64, 128, [700, 1300], [1, 1]),
    "group_of_32": (32, 1, 128, 256, [900], [1]),
    "drafts": (8, 2, 64, 16, [500, 744, 60], [8, 3, 5]),
    "drafts_of_sevens": (28, 4, 128, 64, [300, 95, 610], [5, 9, 2]),
    "a_question": (16, 4, 128, 64, [260, 90], [70, 90]),
    "questions": (28, 4, 128, 32, [700, 300, 64], [130, 37, 64]),
    "a_long_question": (4, 2, 64, 16, [400], [399]),
    "ragged": (28, 4, 128, 64, [2500, 31, 1200, 3, 777], [1, 1, 1, 1, 1]),
    "one_kv_head_of_96": (96, 1, 64, 64, [300, 130], [3, 1]),      # as many heads as the kernel for many rows takes at once
    "one_kv_head_of_130": (130, 1, 128, 64, [200, 77], [2, 1]),    # more
    "more_sequences_than_a_warp": (16, 4, 128, 16, [5 + 29 * i % 190 for i in range(45)], [5 + i % 9 for i in range(45)]),
    "many_groups_a_block": (8, 2, 64, 16, [1 + 83 * i % 300 for i in range(1100)], [7 * (i % 5 > 0) for i in range(1100)]),
    "no_groups": (16, 16, 64, 32, [333, 64, 1000], [1, 2, 1]),
}


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("name", CASES)
def test_what_rows_pay(name, fmt):
    hq, hkv, dim, page, lens, rows = CASES[name]
    w = Weighing(Problem(hq, hkv, dim, fmt, page, lens, rows, seed=len(name)))
    w.run()
    w.check()


@pytest.mark.parametrize("rows", [1, 7, 40, 150])
@pytest.mark.parametrize("causal,strided", [(True, False), (False, True)])
@pytest.mark.parametrize("decay", [0.0, 0.75])
def test_masks_strides_decay_and_new_tokens(rows, causal, strided, decay):
    p = Problem(12, 4, 128, "int8", 32, [190, 300, 157], [rows, 1, max(1, rows - 3)], causal=causal, strided=strided, scale=0.3, seed=5)
    w = Weighing(p, decay=decay, fresh=[190 - rows, 0, 400])
    w.run()
    w.check()


@pytest.mark.parametrize("rows", [1, 3, 40])
def test_rows_that_pay_nothing(rows):
    """A log-sum-exp of -inf is a row that sees no key, whatever the mask says; +inf pays 0."""
    p = Problem(8, 2, 64, "fp8", 16, [100, 20], [rows, 1], causal=False, seed=6)
    w = Weighing(p)
    w.lse[0, ::2] = -math.inf
    w.lse[rows - 1, 1::2] = math.inf
    w.run()
    w.check()


@pytest.mark.parametrize("rows", [1, 2, 24, 100])
def test_rows_and_keys_that_are_not_finite(rows):
    """A query row that is not finite reaches its own KV head's weights of its sequence only, a key that is not finite its own weight."""
    lens = [150, 210]
    p = Problem(8, 2, 128, "int8", 64, lens, [rows, rows], causal=False, seed=9)
    w = Weighing(p)
    w.run()
    clean = w.on_gpu.cpu()
    p.qd = p.q.clone().cuda()
    p.qd[rows, 5, 77] = math.nan                     # sequence 1, KV head 1
    to, slot = w.at[0][0][31], 31 % 64
    p.cache.k_scale[to, 0, slot] = math.nan
    w.on_gpu = w.weights.cuda()
    w.run(q=p.qd)
    dirty = w.on_gpu.cpu()
    off = torch.zeros(dirty.shape, dtype=torch.bool)
    off[to, 0, slot] = True
    off[w.at[1][0], 1, w.at[1][1]] = True
    assert bool(torch.isnan(dirty[off]).all()) and torch.equal(dirty[~off].nan_to_num(-1.0), clean[~off].nan_to_num(-1.0))


@pytest.mark.parametrize("spread", [2.0 ** -40, 30.0])
def test_peaked_and_tiny_logits(spread):
    p = Problem(16, 2, 128, "int8", 32, [500, 77], [2, 1], spread=spread, seed=11)
    w = Weighing(p)
    w.run()
    w.check()


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("power", [2.0 ** 60, 2.0 ** -60])
def test_queries_and_keys_whose_sizes_cancel(rows, power):
    p = Problem(16, 4, 64, "fp8", 32, [300, 45], [rows, 1], spread=1 / power, seed=12)
    p.q = (p.q.double() * power).to(torch.bfloat16)
    p.qd = p.q.cuda()
    w = Weighing(p)
    w.run()
    w.check()


@pytest.mark.parametrize("rows", [2, 60])
def test_rows_behind_the_last_sequence_and_between_streams(rows):
    """q and lse with rows that no sequence has, NaN; two calls at once on streams of their own, on pools of their own."""
    p = Problem(8, 2, 128, "int8", 64, [500, 130], [rows, rows], seed=15)
    w = Weighing(p)
    q = torch.full((2 * rows + 40, 8, 128), math.nan, dtype=torch.bfloat16)
    lse = torch.full((2 * rows + 40, 8), math.nan)
    q[:2 * rows], lse[:2 * rows] = p.q, w.lse
    args = [q.cuda(), lse.cuda(), _cu(p.rows).cuda(), p.tables[0].cuda(), _dev(p.lens)]
    params = p.params(total_q=len(q))
    pools = [w.weights.cuda() for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for pool, stream in zip(pools, streams):
        fastav.fastav_cache_weigh(params, p.cache, pool, *args, device_status=p.status, stream=stream)
    torch.cuda.synchronize()
    w.on_gpu = pools[0]
    w.check()
    assert torch.equal(pools[0].nan_to_num(-1.0), pools[1].nan_to_num(-1.0))


def test_weights_of_the_attention_itself_sum_to_one():
    """Given the log-sum-exp that fastav_attend returns, every row pays 1 per query head: with the prefix's share weighed by a call of its own."""
    lens, rows, plens, groups = [40, 90, 33, 128], [3, 1, 2, 5], [300, 77], [0, 3, 4]
    p = Problem(8, 2, 128, "fp8", 16, lens, rows, prefix_lens=plens, groups=groups, seed=12)
    p.run()
    weights = torch.zeros_like(p.cache.k_scale)
    fastav.fastav_cache_weigh(p.params(), p.cache, weights, p.qd, p.lse, _cu(rows).cuda(), p.tables[0].cuda(), _dev(lens), device_status=p.status)
    group_rows = [sum(rows[a:b]) for a, b in zip(groups, groups[1:])]
    params = fastav.make_attend_params(batch=2, total_q=sum(rows), max_qlen=max(group_rows), num_q_heads=8, max_kv_len=max(plens), q=p.qd, out=p.out,
                                       page_table=p.tables[1])
    fastav.fastav_cache_weigh(params, p.cache, weights, p.qd, p.lse, _cu(group_rows).cuda(), p.tables[1].cuda(), _dev(plens), device_status=p.status)
    assert int(p.status) == 0
    total = weights.double().sum((0, 2)).cpu()                      # per KV head
    # each of rows x G parts is off by its lse's error, 2^-19 or so (tolerances of the attention's tests), and the sums' roundings
    assert float((total / (sum(rows) * 4) - 1).abs().max()) <= 2.0 ** -15


def test_bounds_that_do_not_hold_and_bad_pages():
    p = Problem(8, 2, 64, "int8", 16, [100, 40], [2, 1], seed=13)
    w = Weighing(p)
    w.run(page_table=torch.where(p.tables[0] == p.tables[0][1, 1], 10 ** 6, p.tables[0]).cuda())   # tokens 16 to 31 of sequence 1
    assert int(p.status) == fastav.FASTAV_DEV_BAD_INDEX
    got = w.on_gpu.cpu()
    to, slot = w.at[1][:2]
    assert torch.equal(got[to[16:32], :, slot[16:32]], w.weights[to[16:32], :, slot[16:32]])
    p.status.zero_()
    for over in (dict(max_kv_len=60), dict(max_qlen=1, total_q=3)):
        v = Weighing(p)
        v.run(p.params(**over))
        assert int(p.status) & fastav.FASTAV_DEV_SHAPE_MISMATCH
        v.check(int(p.status), skip=(0,))
        p.status.zero_()
    loose = Weighing(p)                                    # bounds may be loose
    loose.run(p.params(max_kv_len=10 ** 6, max_qlen=3))
    loose.check()


def test_equal_calls_give_equal_bits_on_streams_and_replayed():
    p = Problem(28, 4, 128, "int8", 64, [900, 2000, 31], [1, 12, 9], seed=14)
    w = Weighing(p)
    w.run()
    w.check()
    first = w.on_gpu.clone()
    side, params, args = torch.cuda.Stream(), p.params(), (p.qd, w.lse.cuda(), _cu(p.rows).cuda(), p.tables[0].cuda(), _dev(p.lens))
    start, again = w.weights.cuda(), w.weights.cuda()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        again.copy_(start)
        fastav.fastav_cache_weigh(params, p.cache, again, *args)
    for _ in range(3):
        again.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again.nan_to_num(-1.0), first.nan_to_num(-1.0))


def test_offsets_beyond_32_bits():
    hkv, dim, page = 8, 128, 256
    pages = (5 << 30) // (hkv * dim * page)
    cache = fastav.make_cache(pages, hkv, dim, page)
    weights = torch.zeros_like(cache.k_scale)
    gen = torch.Generator().manual_seed(3)
    for rows in (1, 9):
        n, table = 300, torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32)
        codes = torch.randint(-127, 128, (n, hkv, dim), generator=gen, dtype=torch.int8)
        for t0, at in ((0, pages - 1), (256, pages - 2)):
            m = min(256, n - t0)
            cache.k[at, :, :m] = codes[t0:t0 + m].transpose(0, 1).cuda()
            cache.k_scale[at] = 0.01
            weights[at] = 0
        q = torch.randn(rows, 4 * hkv, dim, generator=gen).to(torch.bfloat16)
        lse = torch.full((rows, 4 * hkv), 5.0)
        params = fastav.make_attend_params(batch=1, total_q=rows, max_qlen=rows, num_q_heads=4 * hkv, max_kv_len=n, q=q, out=q, page_table=table)
        fastav.fastav_cache_weigh(params, cache, weights, q.cuda(), lse.cuda(), _dev([0, rows]), table.cuda(), _dev([n]))
        keys = codes.double() * float(torch.tensor(0.01))
        want, size = ref.weigh(torch.zeros(n, hkv), 1.0, n, q, keys, lse, [n] * rows, dim ** -0.5)
        t = torch.arange(n)
        got = weights[(pages - 1 - t // page).cuda(), :, (t % page).cuda()].cpu().double()
        assert float(((got - want).abs() - size * (12 * 2.0 ** -22 + 2.0 ** -20) - 2.0 ** -24 * 4 * (rows + 1) * want - 4 * rows * 2.0 ** -126).max()) <= 0
