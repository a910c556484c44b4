"""fastav_cache_evict against a plain sort: which tokens stay, and every byte of the cache after it, have to be equal."""
import math

import pytest
import torch

import token_reference as ref
from paper_2601_13143_b200 import fastav

pytestmark = pytest.mark.gpu


class Eviction:
    def __init__(self, lens, keep, hkv, dim, page, fmt="int8", first=0, recent=0, joint=False, apart=False, seed=0, weights=None):
        self.__dict__.update(lens=lens, keep=keep, hkv=hkv, page=page, first=first, recent=recent, joint=joint, apart=apart)
        gen = torch.Generator().manual_seed(seed)
        kept = [max(0, min(k, n)) for k, n in zip(keep, lens)]
        need, need_out = [-(-n // page) for n in lens], [-(-n // page) if apart else 0 for n in kept]
        pages = sum(need) + sum(need_out) + 2
        ids = torch.randperm(pages, generator=gen).to(torch.int32)
        self.table, at = torch.full((len(lens), max(need + [1]) + 1), -3, dtype=torch.int32), 0
        self.out_table = torch.full((len(lens), max(need_out + [1])), -5, dtype=torch.int32)
        for table, needs in ((self.table, need), (self.out_table, need_out)):
            for b, m in enumerate(needs):
                table[b, :m] = ids[at:at + m]
                at += m
        shape = (pages, hkv, page)
        code = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
        self.pools = [torch.randint(-128, 128, (*shape, dim), generator=gen, dtype=torch.int8) for _ in "kv"]
        self.scales = [torch.rand(shape, generator=gen) for _ in "kv"]
        self.weights = torch.exp(2 * torch.randn(shape, generator=gen)) if weights is None else weights(shape, gen)
        self.cache = fastav.KvCache(*[p.view(code).cuda() for p in self.pools], *[s.cuda() for s in self.scales])
        self.on_gpu = self.weights.cuda()
        self.lens_out = torch.full((len(lens),), -9, dtype=torch.int32, device="cuda")
        self.max_keep = max(kept + [0])
        self.idx = torch.full((len(lens), hkv, max(1, self.max_keep)), -9, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def params(self, **over):
        kw = dict(batch=len(self.lens), max_kv_len=max(self.lens), max_keep=self.max_keep, page_table=self.table, out_table=self.out_table if self.apart else None,
                  first=self.first, recent=self.recent, flags=fastav.FASTAV_EVICT_JOINT if self.joint else 0)
        kw.update(over)
        return fastav.make_evict_params(**kw)

    def run(self, params=None, table=None, out_table=None, keep=None, lens=None, idx=True):
        p = params or self.params()
        dev = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731
        ws = torch.full((fastav.fastav_evict_workspace_bytes(p, self.cache),), 0xFF, dtype=torch.uint8, device="cuda")
        out_table = self.out_table if out_table is None else out_table
        fastav.fastav_cache_evict(p, self.cache, self.on_gpu, (self.table if table is None else table).cuda(), dev(self.lens if lens is None else lens),
                                  dev(self.keep if keep is None else keep), self.lens_out, ws, out_table.cuda() if self.apart else None, self.idx if idx else None, self.status)
        torch.cuda.synchronize()

    def expect(self):
        pools, scales, weights = [p.clone() for p in self.pools], [s.clone() for s in self.scales], self.weights.clone()
        idx = torch.full(self.idx.shape, -9, dtype=torch.int32)
        for b, n in enumerate(self.lens):
            t = torch.arange(n)
            w = self.weights[self.table[b].long()[t // self.page], :, t % self.page]          # [n, heads]
            if self.joint:
                w = w.double().sum(1, keepdim=True).float().expand(-1, self.hkv)
            for h in range(self.hkv):
                stay = torch.tensor(ref.survivors(w[:, h], self.keep[b], self.first, self.recent), dtype=torch.int64)
                i = torch.arange(len(stay))
                src, slot = self.table[b].long()[stay // self.page], stay % self.page
                dst, to = (self.out_table if self.apart else self.table)[b].long()[i // self.page], i % self.page
                for new, old in zip((*pools, *scales, weights), (*self.pools, *self.scales, self.weights)):
                    new[dst, h, to] = old[src, h, slot]
                idx[b, h, :len(stay)] = stay.to(torch.int32)
        return pools, scales, weights, idx

    def check(self, status=0, idx=True):
        assert int(self.status) == status
        pools, scales, weights, want = self.expect()
        if idx:
            assert torch.equal(self.idx.cpu(), want)
        assert self.lens_out.tolist() == [max(0, min(k, n)) for k, n in zip(self.keep, self.lens)]
        for got, x in zip((self.cache.k, self.cache.v), pools):
            assert torch.equal(got.view(torch.int8).cpu(), x)
        for got, x in zip((self.cache.k_scale, self.cache.v_scale, self.on_gpu), (*scales, weights)):
            assert torch.equal(got.cpu().view(torch.int32), x.view(torch.int32))


CASES = {
    # lens, keep, heads, dim, page, first, recent
    "one_token": ([1], [1], 1, 64, 16, 0, 0),
    "nothing_stays": ([1, 40], [0, 0], 2, 64, 16, 0, 0),
    "empty_sequences": ([0, 33, 0], [0, 32, 0], 2, 128, 16, 4, 8),
    "all_stay": ([100, 17], [100, 17], 4, 128, 32, 4, 4),
    "one_goes": ([513, 512, 511], [512, 511, 510], 4, 128, 64, 4, 32),
    "one_stays": ([700, 1], [1, 1], 2, 128, 128, 0, 0),
    "odd": ([1000, 333, 64, 65], [501, 77, 63, 2], 3, 64, 16, 1, 3),
    "a_long_one": ([20000], [9001], 2, 128, 256, 16, 300),
    "long_ones": ([9000, 12345], [8999, 400], 8, 64, 64, 0, 64),
    "longer_than_blocks_hold": ([70001], [35000], 1, 64, 256, 4, 64),
    "many": ([60 + 7 * i % 200 for i in range(100)], [30 + 5 * i % 60 for i in range(100)], 8, 64, 16, 2, 10),
    "many_long": ([3000 - 11 * i for i in range(40)], [1500 - 20 * i for i in range(40)], 4, 64, 32, 4, 64),
    "more_than_clusters_at_once": ([300 + i % 50 for i in range(70)], [200] * 70, 8, 64, 64, 0, 16),
}


@pytest.mark.parametrize("joint", [False, True])
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("name", CASES)
def test_survivors_and_the_whole_cache(name, apart, joint):
    lens, keep, hkv, dim, page, first, recent = CASES[name]
    e = Eviction(lens, keep, hkv, dim, page, "fp8" if joint else "int8", first, recent, joint, apart, seed=len(name))
    e.run()
    too_many_stay = any(min(n, first) + min(max(0, n - first), recent) > min(k, n) for n, k in zip(lens, keep))
    e.check((fastav.FASTAV_DEV_PROTECT_OVERFLOW if too_many_stay else 0) | (fastav.FASTAV_DEV_K_CLAMPED if any(k > n for n, k in zip(lens, keep)) else 0))


def _ties(shape, gen):
    return torch.randint(0, 3, shape, generator=gen).float() - 1


def _zeros(shape, gen):
    return torch.where(torch.rand(shape, generator=gen) < 0.5, 0.0, -0.0)


def _odd(shape, gen):
    w = torch.randn(shape, generator=gen) * 1e-38
    pick = torch.rand(shape, generator=gen)
    return torch.where(pick < 0.2, math.nan, torch.where(pick < 0.3, math.inf, torch.where(pick < 0.5, -math.inf, torch.where(pick < 0.6, 1e-45, w))))


def _close(shape, gen):
    return (torch.randint(0, 64, shape, generator=gen) + 0x3F800000).to(torch.int32).view(torch.float32)  # the last bits alone differ


@pytest.mark.parametrize("kind", [_ties, _zeros, _odd, _close])
@pytest.mark.parametrize("n,k", [(40, 21), (3000, 1234), (9000, 8000)])
def test_ties_signs_and_numbers_that_are_none(kind, n, k):
    e = Eviction([n, n // 2], [k, k // 2], 3, 64, 32, first=3, recent=7, weights=kind, seed=n)
    e.run()
    e.check()


def test_joint_weights_are_summed_exactly():
    """Sums that fp32 additions in some order would round differently: one large weight beside many small ones."""
    def weights(shape, gen):
        w = torch.rand(shape, generator=gen) * 2.0 ** -24
        w[:, 0] = 1.0
        return w
    e = Eviction([2000], [777], 8, 64, 16, joint=True, weights=weights)
    e.run()
    e.check()


@pytest.mark.parametrize("apart", [False, True])
def test_protected_tokens_beyond_the_count(apart):
    e = Eviction([50, 10, 200], [20, 4, 100], 2, 64, 16, first=30, recent=40, apart=apart)
    e.run()
    e.check(fastav.FASTAV_DEV_PROTECT_OVERFLOW)


def test_counts_and_lengths_that_do_not_hold():
    e = Eviction([50, 90], [60, -4], 2, 64, 16)
    e.run()
    e.check(fastav.FASTAV_DEV_K_CLAMPED)
    e = Eviction([50, 90], [20, 40], 2, 64, 16)
    e.run(e.params(max_keep=30))
    assert int(e.status) == fastav.FASTAV_DEV_SHAPE_MISMATCH and e.lens_out.tolist() == [20, 30]
    e = Eviction([50, 90], [20, 40], 2, 64, 16)
    e.run(e.params(max_kv_len=60))
    assert int(e.status) == fastav.FASTAV_DEV_SHAPE_MISMATCH and e.lens_out.tolist() == [20, 40] and int(e.idx[1].max()) < 60
    e = Eviction([50, 90], [20, 40], 2, 64, 16)
    e.run(lens=[50, -1])
    assert int(e.status) & fastav.FASTAV_DEV_SHAPE_MISMATCH and e.lens_out.tolist() == [20, 0]


def test_pages_that_are_none():
    e = Eviction([64], [40], 2, 64, 16, apart=True)
    table = e.table.clone()
    table[0, 1] = 10 ** 6
    e.run(table=table)
    assert int(e.status) == fastav.FASTAV_DEV_BAD_INDEX and e.lens_out.tolist() == [40]
    kept = e.idx.cpu()
    assert not bool(((kept >= 16) & (kept < 32)).any())                              # they rank lowest
    e = Eviction([64], [60], 2, 64, 16, apart=True)                                  # ... and are left out where they have to stay
    e.run(table=table.new_tensor([[int(e.table[0, 0]), -1, int(e.table[0, 2]), int(e.table[0, 3]), 0]]))
    assert int(e.status) == fastav.FASTAV_DEV_BAD_INDEX
    e = Eviction([64], [40], 2, 64, 16, apart=True)
    out = e.out_table.clone()
    out[0, 1] = -1
    before = [x.clone() for x in (e.cache.k, e.cache.k_scale, e.on_gpu)]
    e.run(out_table=out)
    assert int(e.status) == fastav.FASTAV_DEV_BAD_INDEX
    for x, y in zip(before, (e.cache.k, e.cache.k_scale, e.on_gpu)):
        page = int(e.out_table[0, 1])
        assert torch.equal(x[page].view(torch.int8), y[page].view(torch.int8))


def test_sequences_may_share_pages_that_nothing_is_written_to():
    """Two sequences with the same first pages, compacted into pages of their own; without the list of survivors."""
    e = Eviction([100, 100], [30, 50], 2, 128, 16, apart=True)
    e.table[1, :4] = e.table[0, :4]
    e.run(idx=False)
    e.check(idx=False)


def test_again_and_again_in_place():
    """One token less per step, nothing new between: ten evictions leave what one does."""
    e = Eviction([300], [299], 2, 64, 16, first=4, recent=8)
    want_first = [ref.survivors(e.weights[e.table[0].long()[torch.arange(300) // 16], h, torch.arange(300) % 16], 290, 4, 8) for h in range(2)]
    for n in range(300, 290, -1):
        e.run(lens=[n], keep=[n - 1])
        assert e.lens_out.tolist() == [n - 1]
    i = torch.arange(290)
    for h in range(2):
        got = e.on_gpu.cpu()[e.table[0].long()[i // 16], h, i % 16]
        w = e.weights[e.table[0].long()[torch.arange(300) // 16], h, torch.arange(300) % 16]
        assert torch.equal(got, w[torch.tensor(want_first[h])])


def test_streams_and_replay():
    e = Eviction([2000, 900], [700, 450], 4, 128, 64, apart=True, first=2, recent=9)
    e.run()
    e.check()
    params, side = e.params(), torch.cuda.Stream()
    ws = torch.empty(fastav.fastav_evict_workspace_bytes(params, e.cache), dtype=torch.uint8, device="cuda")
    dev = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    table, out_table, lens, keep, counts = e.table.cuda(), e.out_table.cuda(), dev(e.lens), dev(e.keep), dev([0, 0])
    start = e.weights.cuda()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        e.on_gpu.copy_(start)
        counts.copy_(keep)
        fastav.fastav_cache_evict(params, e.cache, e.on_gpu, table, lens, counts, e.lens_out, ws, out_table, e.idx, e.status)
    for seed in (5, 6):
        e.weights = torch.exp(torch.randn(e.weights.shape, generator=torch.Generator().manual_seed(seed)))
        start.copy_(e.weights.cuda())
        e.cache.k_scale.copy_(e.scales[0].cuda())
        e.cache.v_scale.copy_(e.scales[1].cuda())
        for x, p in zip((e.cache.k, e.cache.v), e.pools):
            x.copy_(p.cuda())
        graph.replay()
        torch.cuda.synchronize()
        e.check()


def test_offsets_beyond_32_bits():
    hkv, dim, page = 8, 128, 256
    pages = (5 << 30) // (hkv * dim * page)
    cache = fastav.make_cache(pages, hkv, dim, page)
    weights = torch.rand(cache.k_scale.shape, device="cuda")
    table = torch.tensor([[pages - 1, pages - 2, pages - 4]], dtype=torch.int32)
    n, k, t = 700, 300, torch.arange(700)
    at, slot = table[0].long()[t // page].cuda(), (t % page).cuda()
    rows = torch.randint(-128, 128, (n, hkv, dim), dtype=torch.int8, device="cuda")
    cache.k[at, :, slot] = rows
    cache.v[at, :, slot] = rows.flip(2)
    w = weights[at, :, slot].clone()
    lens, out = torch.tensor([n], dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    p = fastav.make_evict_params(batch=1, max_kv_len=n, max_keep=k, page_table=table)
    ws = torch.empty(fastav.fastav_evict_workspace_bytes(p, cache), dtype=torch.uint8, device="cuda")
    fastav.fastav_cache_evict(p, cache, weights, table.cuda(), lens, torch.tensor([k], dtype=torch.int32).cuda(), out, ws)
    for h in range(hkv):
        stay = torch.tensor(ref.survivors(w[:, h].cpu(), k, 0, 0)).cuda()
        assert torch.equal(cache.k[at[:k], h, slot[:k]], rows[stay, h]) and torch.equal(cache.v[at[:k], h, slot[:k]], rows.flip(2)[stay, h])
        assert torch.equal(weights[at[:k], h, slot[:k]], w[stay, h])
