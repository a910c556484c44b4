"""fastav_attend against the definition in 64 bits.

Tolerances.  The logits are sums of exact products in fp32: d / 16 steps of the matrix unit and a few products, each off by at most 2^-22 of
the sum of magnitudes.  The weights are rounded to f16 (2^-11), their exponentials are good to 2^-21; the output is rounded to bf16 (2^-9).  So
    |lse - ref| <= B (d / 16 + 4) 2^-22 + 2^-20 (1 + |ref|),   B = largest sum_i |q_i k_ji| scale over the visible keys
    |out - ref| <= 2^-8 |ref| + (2^-10 + 2 (B (d / 16 + 4) 2^-22)) sum_j p_j |v_j| + 2^-36 n max_j (p_j max_i |v_ji|)
where the last term is what f16 cannot hold: a row's largest weight (times the value's scale) is laid on 2^11 at least, so small ones are off by up to
2^-25 of a unit, 2^-36 of the largest, each times a code; it shows where the tokens that matter have a code of exactly 0."""
import math

import pytest
import torch

import cache_reference as ref
from paper_2601_13143_b200 import fastav

pytestmark = pytest.mark.gpu
CODE = {"int8": torch.int8, "fp8": torch.float8_e4m3fn}


def _cu(counts):
    return torch.tensor([0] + list(counts), dtype=torch.int64).cumsum(0).to(torch.int32)


class Problem:
    def __init__(self, hq, hkv, dim, fmt, page, lens, rows, causal=True, prefix_lens=(), groups=(), seed=0, spread=1.0, scale=0.0, strided=False):
        self.__dict__.update(hq=hq, hkv=hkv, dim=dim, fmt=fmt, page=page, lens=lens, rows=rows, causal=causal, prefix_lens=list(prefix_lens), groups=list(groups),
                             scale=scale)
        gen = self.gen = torch.Generator().manual_seed(seed)
        code = CODE[fmt]
        need = [[-(-n // page) for n in l] for l in (lens, self.prefix_lens)]
        pages = sum(map(sum, need)) + 1
        ids = torch.randperm(pages, generator=gen).to(torch.int32)
        # what no sequence's token fills is hostile: NaN codes or extreme ones, scales that are NaN or infinite
        k_pool = torch.full((pages, hkv, page, dim), 0x7F, dtype=torch.int8)
        v_pool = k_pool.clone()
        k_scale = torch.full((pages, hkv, page), math.nan)
        v_scale = torch.full((pages, hkv, page), math.inf)
        tables, self.tokens, at = [], [], 0
        for l, nd in zip((lens, self.prefix_lens), need):
            table = torch.full((max(len(l), 1), max(nd + [0]) + 2), -1, dtype=torch.int32)
            for b, n in enumerate(l):
                table[b, :nd[b]] = ids[at:at + nd[b]]
                at += nd[b]
                pair = []
                for pool, scale_pool in ((k_pool, k_scale), (v_pool, v_scale)):
                    x = torch.randn(n, hkv, dim, generator=gen) * torch.exp2(torch.randint(-2, 3, (n, hkv, 1), generator=gen).float())
                    if pool is k_pool:
                        x *= spread
                    c, s = ref.quantise(x.to(torch.bfloat16), code)
                    t = torch.arange(n)
                    pool[table[b].long()[t // page], :, t % page] = c.float().to(code).view(torch.int8)
                    scale_pool[table[b].long()[t // page], :, t % page] = s
                    pair.append(c * s.double()[..., None])
                self.tokens.append(pair)
            tables.append(table)
        self.tables = tables
        self.cache = fastav.KvCache(k_pool.view(code).cuda(), v_pool.view(code).cuda(), k_scale.cuda(), v_scale.cuda())
        self.total = sum(rows)
        self.q = (torch.randn(self.total, hq, dim, generator=gen) * torch.exp2(torch.randint(-1, 2, (self.total, hq, 1), generator=gen).float())).to(torch.bfloat16)
        if strided:  # heads of a packed projection, rows of a wider output
            wide = torch.full((self.total, hq + 3, dim + 8), 5.0, dtype=torch.bfloat16, device="cuda")
            wide[:, 1:hq + 1, 8:] = self.q.cuda()
            self.qd = wide[:, 1:hq + 1, 8:]
            self.out = torch.full((self.total, hq + 2, dim + 16), 7.0, dtype=torch.bfloat16, device="cuda")[:, 1:hq + 1, 8:dim + 8]
        else:
            self.qd = self.q.cuda()
            self.out = torch.full((self.total, hq, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((self.total, hq), 7.0, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def sees(self, b):
        n, r = self.lens[b], self.rows[b]
        return [n - r + i + 1 if self.causal else n for i in range(r)]

    def params(self, **over):
        g = self.groups
        kw = dict(batch=len(self.lens), total_q=self.total, max_qlen=max(self.rows), num_q_heads=self.hq, max_kv_len=max(self.lens), q=self.qd, out=self.out,
                  page_table=self.tables[0], prefix_table=self.tables[1] if self.prefix_lens else None, max_prefix_len=max(self.prefix_lens, default=0),
                  max_prefix_q=max((sum(self.rows[a:b]) for a, b in zip(g, g[1:])), default=0), softmax_scale=self.scale,
                  flags=fastav.FASTAV_CAUSAL if self.causal else 0)
        kw.update(over)
        return fastav.make_attend_params(**kw)

    def run(self, params=None, stream=None, workspace=None):
        p = params or self.params()
        ws = workspace if workspace is not None else torch.full((fastav.fastav_attend_workspace_bytes(p, self.cache),), 0xFF, dtype=torch.uint8, device="cuda")
        dev = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731
        more = dict(cu_prefix=dev(self.groups), prefix_table=self.tables[1].cuda(), prefix_lens=dev(self.prefix_lens)) if self.prefix_lens else {}
        fastav.fastav_attend(p, self.cache, self.qd, _cu(self.rows).cuda(), self.tables[0].cuda(), dev(self.lens), self.out, ws, lse_out_opt=self.lse,
                             device_status=self.status, stream=stream, **more)
        torch.cuda.synchronize()

    def check(self, status=0, skip=()):
        assert int(self.status) == status
        out, lse = self.out.cpu().double(), self.lse.cpu().double()
        cu = _cu(self.rows).tolist()
        scale = self.scale if self.scale > 0 else 1 / math.sqrt(self.dim)
        for b in range(len(self.lens)):
            if b in skip or self.rows[b] == 0:
                continue
            k, v = self.tokens[b]
            sees = self.sees(b)
            for p, n in enumerate(self.prefix_lens):
                if self.groups[p] <= b < self.groups[p + 1]:
                    pk, pv = self.tokens[len(self.lens) + p]
                    k, v = torch.cat([pk, k]), torch.cat([pv, v])
                    sees = [max(s, 0) + n for s in sees]
            want, wlse, mass, size, most = ref.attend(self.q[cu[b]:cu[b + 1]], k, v, sees, scale)
            got, glse = out[cu[b]:cu[b + 1]], lse[cu[b]:cu[b + 1]]
            none = torch.isinf(wlse)
            assert torch.equal(none, torch.isinf(glse)) and bool((glse[none] < 0).all()) and bool((got[none] == 0).all())
            off = size * (self.dim / 16 + 4) * 2.0 ** -22
            bad = (glse - wlse).abs()[~none] - (off + 2.0 ** -20 * (1 + wlse.abs()))[~none]
            assert bad.numel() == 0 or float(bad.max()) <= 0, (b, float(bad.max()))
            excess = (got - want).abs() - (2.0 ** -8 * want.abs() + (2.0 ** -10 + 2 * off)[..., None] * mass + 2.0 ** -36 * most[..., None])
            assert float(excess.max()) <= 0, (b, float(excess.max()))


CASES = {
    # hq, hkv, dim, page, lens, rows
    "one_key": (8, 2, 64, 16, [1], [1]),
    "lengths_around_a_granule": (28, 4, 128, 16, [31, 32, 33, 1, 64, 65, 17, 15, 16], [1] * 9),
    "no_keys_and_no_rows": (8, 2, 128, 64, [0, 5, 0, 40], [1, 0, 0, 2]),
    "more_rows_than_keys": (8, 2, 128, 32, [3, 1, 0], [7, 4, 3]),
    "many_short": (32, 8, 128, 16, [7 + 13 * i % 61 for i in range(150)], [1] * 150),
    "one_head_long": (1, 1, 128, 64, [9001], [1]),
    "group_of_16": (32, 2, 64, 128, [700, 1300], [1, 1]),
    "group_of_32": (32, 1, 128, 256, [900], [1]),
    "drafts": (8, 2, 64, 16, [500, 744, 60], [8, 3, 5]),
    "drafts_of_sevens": (28, 4, 128, 64, [300, 95, 610], [5, 9, 2]),
    "a_question": (16, 4, 128, 64, [260, 90], [70, 90]),
    "ragged": (28, 4, 128, 64, [2500, 31, 1200, 3, 777], [1, 1, 1, 1, 1]),
    "no_groups": (16, 16, 64, 32, [333, 64, 1000], [1, 2, 1]),
}


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("name", CASES)
def test_own_tokens(name, fmt):
    hq, hkv, dim, page, lens, rows = CASES[name]
    p = Problem(hq, hkv, dim, fmt, page, lens, rows, seed=len(name))
    p.run()
    p.check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("strided", [True, False])
def test_mask_strides_and_scale(causal, strided):
    p = Problem(12, 4, 128, "int8", 32, [40, 100, 7], [6, 1, 7], causal=causal, strided=strided, scale=0.3, seed=5)
    p.run()
    p.check()
    if strided:
        whole = p.out.as_strided((p.total, p.hq + 2, p.dim + 16), (p.out.stride(0), p.out.stride(1), 1), 0)
        untouched = torch.ones_like(whole, dtype=torch.bool)
        untouched[:, 1:p.hq + 1, 8:p.dim + 8] = False
        assert bool((whole[untouched] == 7).all())


SHARED = {
    # hq, hkv, dim, page, lens, rows, prefix lens, groups
    "one_prefix": (32, 8, 128, 64, [20, 100, 1, 60], [1, 1, 1, 1], [700], [0, 4]),
    "three_prefixes_and_one_without": (28, 4, 128, 32, [20, 33, 64, 5, 9, 40], [1, 3, 2, 1, 8, 1], [300, 1, 129], [0, 2, 3, 5]),
    "prefix_alone": (8, 2, 64, 16, [0, 0, 3], [2, 1, 1], [95], [0, 3]),
    "an_empty_prefix": (8, 2, 64, 16, [10, 20], [1, 1], [0, 50], [0, 1, 2]),
    "nothing_at_all": (8, 2, 64, 16, [0, 20], [1, 1], [0], [0, 2]),
    "many_rows": (32, 8, 128, 64, [64, 70, 90, 33], [40, 70, 33, 20], [600], [0, 4]),
    "many_sequences": (28, 4, 128, 64, [3 + 7 * i % 50 for i in range(70)], [1 + i % 3 for i in range(70)], [513], [0, 70]),
    "rows_that_fill_tiles": (16, 4, 64, 128, [128] * 4, [32] * 4, [1000], [0, 4]),
}


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("name", SHARED)
def test_shared_prefixes(name, fmt):
    hq, hkv, dim, page, lens, rows, prefix_lens, groups = SHARED[name]
    p = Problem(hq, hkv, dim, fmt, page, lens, [min(r, max(n, r)) for r, n in zip(rows, lens)], prefix_lens=prefix_lens, groups=groups, seed=len(name))
    p.run()
    p.check()


@pytest.mark.parametrize("spread", [0.0, 30.0])
def test_flat_and_peaked_weights(spread):
    """Equal logits, and logits of which one outweighs all others, in every order of appearance (the running maximum moves)."""
    p = Problem(8, 2, 128, "int8", 64, [1000, 300], [1, 2], spread=spread, seed=3)
    p.run()
    p.check()


@pytest.mark.parametrize("first", [1e-9, 1e9])
def test_values_of_very_different_size(first):
    """Half of the tokens' values are 10^9 times as large as the others', the larger ones first or last."""
    p = Problem(8, 2, 128, "fp8", 64, [640], [1], seed=4)
    k, v = p.tokens[0]
    t = torch.arange(320)
    to = p.tables[0][0].long()[t // 64]
    scale = p.cache.v_scale.cpu()
    scale[to, :, t % 64] *= first
    v[:320] = p.cache.v.float().cpu().double()[to, :, t % 64] * scale[to, :, t % 64].double()[..., None]
    p.cache.v_scale.copy_(scale)
    p.run()
    p.check()


def test_equal_calls_give_equal_bits_and_leave_nothing_behind():
    p = Problem(28, 4, 128, "fp8", 64, [1500, 70, 333], [1, 4, 2], prefix_lens=[800], groups=[0, 2], seed=9)
    ws = torch.empty(fastav.fastav_attend_workspace_bytes(p.params(), p.cache), dtype=torch.uint8, device="cuda")
    seen = []
    for i in range(4):
        ws.fill_(0xFF if i % 2 else 0)
        p.out.fill_(0)
        p.run(workspace=ws)
        seen.append((p.out.clone(), p.lse.clone()))
    p.check()
    assert all(torch.equal(a, seen[0][0]) and torch.equal(b, seen[0][1]) for a, b in seen)


def test_host_bounds_may_be_larger_and_too_small_ones_are_reported():
    p = Problem(8, 2, 128, "int8", 64, [200, 90], [2, 1], seed=10)
    p.run(p.params(max_qlen=3, max_kv_len=4096))
    p.check()
    p.run(p.params(max_kv_len=100))
    assert int(p.status) == fastav.FASTAV_DEV_SHAPE_MISMATCH


def test_a_page_outside_the_pool_is_reported_and_harms_its_sequence_only():
    p = Problem(8, 2, 128, "int8", 64, [200, 90, 70], [1, 1, 1], seed=11)
    p.tables[0][1, 1] = 1 << 30
    p.run()
    p.check(fastav.FASTAV_DEV_BAD_INDEX, skip=(1,))


def test_not_finite_rows_reach_the_rows_that_see_them_only():
    p = Problem(8, 2, 128, "fp8", 64, [100], [4], seed=12)
    page, slot = int(p.tables[0][0, 98 // 64]), 98 % 64   # seen by rows 2 and 3 (they see 99 and 100 tokens)
    p.cache.k_scale[page, 1, slot] = math.nan
    p.run()
    out, lse = p.out.cpu(), p.lse.cpu()
    assert bool(torch.isfinite(out[:2].float()).all()) and bool(torch.isfinite(lse[:2]).all()) and bool(torch.isfinite(out[2:, :4].float()).all())
    assert bool(torch.isnan(out[2:, 4:].float()).all()) and bool(torch.isnan(lse[2:, 4:]).all())


def test_its_log_sum_exp_serves_the_score_call():
    """Cache written from bf16 keys whose values are codes (no rounding), then fastav_score with the reported lse: weights that sum to 1."""
    hq, hkv, dim, n = 8, 2, 128, 500
    gen = torch.Generator().manual_seed(2)
    k = torch.randint(-126, 127, (n, hkv, dim), generator=gen).float()
    k[..., 0] = 127
    k = (k / 64).to(torch.bfloat16).cuda()
    q = torch.randn(1, hq, dim, generator=gen).to(torch.bfloat16).cuda()
    cache = fastav.make_cache(8, hkv, dim)
    table = torch.arange(8, dtype=torch.int32).cuda()[None]
    cu, cu_q = _cu([n]).cuda(), _cu([1]).cuda()
    params = fastav.make_params(batch=1, total_tokens=n, max_seqlen=n, total_q=1, max_qlen=1, total_keep=0, max_keep=0, num_q_heads=hq, num_kv_heads=hkv,
                                head_dim=dim, hidden=0, q=q, k=k, v=k, flags=fastav.FASTAV_CAUSAL)
    fastav.fastav_cache_write(params, cache, k, k, cu, None, None, table)
    out, lse = torch.empty_like(q), torch.empty(1, hq, device="cuda")
    ap = fastav.make_attend_params(batch=1, total_q=1, max_qlen=1, num_q_heads=hq, max_kv_len=n, q=q, out=out, page_table=table, flags=fastav.FASTAV_CAUSAL)
    ws = torch.empty(fastav.fastav_attend_workspace_bytes(ap, cache), dtype=torch.uint8, device="cuda")
    fastav.fastav_attend(ap, cache, q, cu_q, table, torch.tensor([n], dtype=torch.int32).cuda(), out, ws, lse_out_opt=lse)
    scores, ws2 = torch.empty(n, device="cuda"), torch.empty(fastav.fastav_workspace_bytes(params), dtype=torch.uint8, device="cuda")
    q_idx = torch.tensor([n - 1], dtype=torch.int32).cuda()
    fastav.fastav_score(params, q, q_idx, cu_q, k, cu, scores, ws2, lse_opt=lse)
    assert abs(float(scores.double().sum()) - 1) < 2e-4
    own = torch.empty_like(scores)
    fastav.fastav_score(params, q, q_idx, cu_q, k, cu, own, ws2)
    assert float((scores - own).abs().max()) <= 2e-4 * float(own.max())


def test_offsets_beyond_32_bits():
    hq, hkv, dim, page = 16, 8, 128, 256
    pages = (5 << 30) // (hkv * dim * page)
    cache = fastav.make_cache(pages, hkv, dim, page)
    p = Problem(hq, hkv, dim, "int8", page, [600], [1], seed=13)
    table = torch.tensor([[pages - 1, 3, pages - 2, 0]], dtype=torch.int32)
    for i in range(3):
        for name in ("k", "v", "k_scale", "v_scale"):
            getattr(cache, name)[int(table[0, i])] = getattr(p.cache, name)[int(p.tables[0][0, i])]
    p.cache, p.tables[0] = cache, table
    p.run()
    p.check()


def test_the_largest_batch():
    """4,096 entries: 4,094 sequences of 0 to 6 tokens and two prefixes."""
    lens, rows = [i % 7 for i in range(4094)], [1] * 4094
    p = Problem(2, 1, 64, "int8", 16, lens, rows, prefix_lens=[3, 1], groups=[0, 2000, 4000], seed=14)
    p.run()
    p.check()


@pytest.mark.parametrize("entries", [2998, 3002])
def test_many_rows_of_more_sequences_than_a_block_lists_in_shared_memory(entries):
    """Two rows of 32 heads on one KV head each; up to 3,000 entries are listed in shared memory."""
    lens, rows = [i % 9 for i in range(entries - 1)], [2] * (entries - 1)
    p = Problem(32, 1, 64, "fp8", 16, lens, rows, prefix_lens=[5], groups=[3, 2001], seed=15)
    p.run()
    p.check()


MIXES = [  # few rows only, many rows only, both side by side, short ones, many partial results
    dict(hq=28, hkv=4, dim=128, fmt="int8", page=64, lens=[3000, 40], rows=[1, 1]),
    dict(hq=16, hkv=4, dim=128, fmt="fp8", page=32, lens=[700, 300], rows=[40, 64]),
    dict(hq=32, hkv=8, dim=128, fmt="int8", page=64, lens=[30, 60, 7] * 6, rows=[1] * 18, prefix_lens=[2000], groups=[0, 18]),
    dict(hq=8, hkv=2, dim=64, fmt="fp8", page=16, lens=[5, 70], rows=[2, 3]),
    dict(hq=32, hkv=1, dim=64, fmt="int8", page=128, lens=[5000], rows=[4]),
]


@pytest.mark.parametrize("flags", [0, fastav.FASTAV_CHAIN_CALLS])
def test_calls_one_behind_the_other_do_not_disturb_each_other(flags):
    """The same calls alone, and in a row without a pause on one workspace, give the same bits."""
    problems = [Problem(seed=20 + i, **m) for i, m in enumerate(MIXES)]
    alone = []
    for p in problems:
        p.run()
        p.check()
        alone.append((p.out.clone(), p.lse.clone()))
    params = [p.params(flags=fastav.FASTAV_CAUSAL | flags) for p in problems]
    ws = torch.full((max(fastav.fastav_attend_workspace_bytes(q, p.cache) for p, q in zip(problems, params)),), 0xFF, dtype=torch.uint8, device="cuda")
    dev = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    arrays = [dict(cu=_cu(p.rows).cuda(), table=p.tables[0].cuda(), lens=dev(p.lens),
                   more=dict(cu_prefix=dev(p.groups), prefix_table=p.tables[1].cuda(), prefix_lens=dev(p.prefix_lens)) if p.prefix_lens else {}) for p in problems]
    torch.cuda.synchronize()
    outs = []
    for turn in range(6):
        for i in [(3 * j + turn) % len(problems) for j in range(len(problems))]:
            p, q, a = problems[i], params[i], arrays[i]
            out, lse = torch.full_like(p.out, 9.0), torch.full_like(p.lse, 9.0)
            fastav.fastav_attend(q, p.cache, p.qd, a["cu"], a["table"], a["lens"], out, ws, lse_out_opt=lse, device_status=p.status, **a["more"])
            outs.append((i, out, lse))
    torch.cuda.synchronize()
    for i, out, lse in outs:
        assert torch.equal(out, alone[i][0]) and torch.equal(lse, alone[i][1]), i
    assert all(int(p.status) == 0 for p in problems)


def test_lengths_and_rows_that_earlier_work_on_the_stream_writes():
    """kv_lens, the page table and q made by kernels right before the call, on a stream of the caller's."""
    p = Problem(28, 4, 128, "int8", 64, [900, 333], [2, 1], prefix_lens=[600], groups=[0, 2], seed=30)
    p.run()
    want, wlse = p.out.clone(), p.lse.clone()
    params = p.params()
    ws = torch.empty(fastav.fastav_attend_workspace_bytes(params, p.cache), dtype=torch.uint8, device="cuda")
    dev = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    cu, lens, groups, plens, table, ptable = _cu(p.rows).cuda(), dev(p.lens), dev(p.groups), dev(p.prefix_lens), p.tables[0].cuda(), p.tables[1].cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for i in range(8):
            p.out.fill_(0)
            lens2, table2, q2, plens2 = lens + i, table + 0, p.qd + 0, plens - i
            lens2 -= i
            plens2 += i
            fastav.fastav_attend(params, p.cache, q2, cu, table2, lens2, p.out, ws, cu_prefix=groups, prefix_table=ptable + 0, prefix_lens=plens2, lse_out_opt=p.lse,
                                 device_status=p.status)
            got = p.out.clone()
            side.synchronize()
            assert torch.equal(got, want) and torch.equal(p.lse, wlse) and int(p.status) == 0
