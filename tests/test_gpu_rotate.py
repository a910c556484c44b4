"""fastav_rotate and fastav_rotate_write against the definition in 64 bits.

Tolerances.  A turn's fraction is rounded to 24 bits (2^-25 of half a turn, 2^-23 rad), sine and cosine to 2^-22, the norm (16 squares a lane, three to four sums of
lanes, a reciprocal root) and its two products to 2^-21, the rotation's products and sums to 2^-23 each: together less than 2^-19 of the pair's magnitude
|a| + |b|.  Then one rounding: to bf16 half a step, 2^-8 of the value; to a code half of its step (int8 1/2; e4m3 2^-4 of the value, 2^-10 at least)."""
import math

import pytest
import torch

import cache_reference as cref
import token_reference as ref
from paper_2601_13143_b200 import fastav
from test_gpu_cache import FORMATS, POISON, _cache, _cu, _tables

pytestmark = pytest.mark.gpu
FP32 = 2.0 ** -19


def _values(gen, n, heads, dim):
    return (torch.randn(n, heads, dim, generator=gen) * torch.exp2(torch.randint(-6, 7, (n, heads, 1), generator=gen).float())).to(torch.bfloat16)


def _positions(gen, axes, n, most=200000):
    return torch.randint(0, most, (axes, n), generator=gen, dtype=torch.int64).to(torch.int32)


def _near(got, want, size):
    excess = (got.cpu().double() - want).abs() - (2.0 ** -8 * want.abs() + FP32 * size + 1e-38)
    assert float(excess.max()) <= 0, float(excess.max())


CASES = {
    # tokens, hq, hkv, dim, rotary, axes, interleaved, q normed, k normed, packed
    "one_token": (1, 28, 4, 128, 128, 3, False, True, True, False),
    "one_head": (7, 1, 1, 64, 64, 1, False, False, False, False),
    "half_of_a_small_head": (33, 8, 2, 64, 32, 1, True, True, False, True),
    "a_quarter": (20, 8, 2, 64, 16, 2, False, False, True, True),
    "three_quarters": (19, 5, 3, 128, 96, 4, True, True, True, False),
    "no_rotation": (11, 4, 4, 128, 0, 1, False, True, True, True),
    "nothing_but_a_copy": (11, 4, 4, 64, 0, 1, False, False, False, True),
    "decode": (32, 28, 4, 128, 128, 1, True, True, True, False),
    "prompt": (3000, 28, 4, 128, 128, 3, False, True, True, True),
    "long_prompt": (9001, 8, 2, 64, 64, 3, False, False, False, True),
    "many_heads": (5, 70, 70, 128, 128, 3, False, True, True, True),
    "odd_heads": (2001, 7, 1, 128, 64, 2, True, False, True, True),
}


def _make(name, seed=0):
    n, hq, hkv, dim, rotary, axes, interleaved, qn, kn, packed = CASES[name]
    gen = torch.Generator().manual_seed(seed + len(name))
    q, k, v = _values(gen, n, hq, dim), _values(gen, n, hkv, dim), _values(gen, n, hkv, dim)
    pos = _positions(gen, axes, n)
    freq = [10000.0 ** (-2.0 * i / max(rotary, 1)) for i in range(rotary // 2)]
    axis = [i * 7 % axes for i in range(rotary // 2)]
    norms = [(1 + 0.3 * torch.randn(dim, generator=gen)).to(torch.bfloat16) if given else None for given in (qn, kn)]
    dev = [x.cuda() for x in (q, k, v)]
    if packed:
        whole = torch.full((n, hq + 2 * hkv + 1, dim + 8), 9.0, dtype=torch.bfloat16, device="cuda")
        parts = [whole[:, a:b, 8:] for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv + 1, hq + 2 * hkv + 1))]
        for to, x in zip(parts, dev):
            to.copy_(x)
        dev = parts
    want = [ref.turned(x, pos, freq, axis, interleaved, norm, 1e-5 if norm is not None else 0.0) for x, norm in ((q, norms[0]), (k, norms[1]))]
    return q, k, v, dev, pos, freq, axis, interleaved, norms, want


def _cuda(x):
    return None if x is None else x.cuda()


@pytest.mark.parametrize("name", CASES)
def test_prompts(name):
    q, k, v, (qd, kd, vd), pos, freq, axis, interleaved, norms, want = _make(name)
    n, hq, dim = q.shape
    wide = torch.full((n, hq + k.shape[1] + 1, dim), 3.0, dtype=torch.bfloat16, device="cuda")
    qo, ko = wide[:, :hq], wide[:, hq + 1:]
    params = fastav.make_rotate_params(q=qd, k=kd, q_out=qo, k_out=ko, pos=pos, frequencies=freq, axis=axis, interleaved=interleaved, norm_eps=1e-5)
    fastav.fastav_rotate(params, qd, kd, pos.cuda(), qo, ko, *map(_cuda, norms))
    _near(qo, *want[0])
    _near(ko, *want[1])
    assert bool((wide[:, hq] == 3).all()) and torch.equal(qd.cpu(), q)
    # one side alone; the other way of laying positions down
    alone = torch.empty_like(kd)
    by_token = pos.T.contiguous().cuda()
    params = fastav.make_rotate_params(k=kd, k_out=alone, pos=by_token.T, frequencies=freq, axis=axis, interleaved=interleaved, norm_eps=1e-5)
    fastav.fastav_rotate(params, None, kd, by_token, None, alone, None, _cuda(norms[1]))
    assert torch.equal(alone, ko)
    # in place
    params = fastav.make_rotate_params(q=qd, k=kd, q_out=qd, k_out=kd, pos=pos, frequencies=freq, axis=axis, interleaved=interleaved, norm_eps=1e-5)
    fastav.fastav_rotate(params, qd, kd, pos.cuda(), qd, kd, *map(_cuda, norms))
    assert torch.equal(qd, qo) and torch.equal(kd, ko) and torch.equal(vd.cpu(), v)


def _check_rows(cache, fmt, table, page, rows):
    """rows: [(sequence, first token, K before rounding and the magnitude of its pairs, V)]; all other places are as they were."""
    code = FORMATS[fmt][1]
    untouched = torch.ones(cache.k_scale.shape, dtype=torch.bool)
    codes = [x.cpu().view(code).double() if fmt == "fp8" else x.cpu().double() for x in (cache.k, cache.v)]
    scales = [x.cpu().double() for x in (cache.k_scale, cache.v_scale)]
    for b, first, (kx, size), vx in rows:
        at = first + torch.arange(len(vx))
        to, slot = table[b].long()[at // page], at % page
        untouched[to, :, slot] = False
        want, scale = cref.quantise(vx, code)
        assert torch.equal(codes[1][to, :, slot], want) and torch.equal(scales[1][to, :, slot].float(), scale)
        got, got_scale, top = codes[0][to, :, slot], scales[0][to, :, slot], kx.abs().amax(-1)
        largest = cref.LARGEST[code]
        assert float(((got_scale - top / largest).abs() - (2 * FP32 * size.amax(-1) / largest + 1e-44)).max()) <= 0
        y, err = kx * (largest / top.clamp(min=1e-300))[..., None], 2 * FP32 * size * (largest / top.clamp(min=1e-300))[..., None] + 2 * FP32 * largest
        half = 0.5 if fmt == "int8" else torch.maximum(y.abs() * 2.0 ** -4, torch.full_like(y, 2.0 ** -10))
        assert float(((got - y).abs() - half - err)[top > 0].max()) <= 0
        assert bool((got[top == 0] == 0).all())
    raw = [x.view(torch.int8).cpu() for x in (cache.k, cache.v)]
    assert all(bool((x[untouched] == POISON).all()) for x in raw)
    assert bool((cache.k_scale.cpu()[untouched] == -3).all()) and bool((cache.v_scale.cpu()[untouched] == -5).all())


WRITES = {
    # case, lengths, first tokens, page
    "one_token": ([1], [40], 16),
    "half_of_a_small_head": ([1, 0, 30, 2], [0, 5, 7, 31], 32),
    "no_rotation": ([11], [0], 64),
    "decode": ([1] * 32, [(37 * i) % 600 for i in range(32)], 16),
    "prompt": ([1000, 1, 0, 1999], [0, 15, 3, 130], 128),
    "odd_heads": ([2001], [1], 256),
    "many_heads": ([2, 3], [0, 0], 64),
}


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("name", WRITES)
def test_new_tokens_go_into_the_cache(name, fmt):
    lens, start, page = WRITES[name]
    q, k, v, (qd, kd, vd), pos, freq, axis, interleaved, norms, want = _make(name, 50)
    hkv, dim = k.shape[1:]
    table, pages = _tables(torch.Generator().manual_seed(4), [s + n for s, n in zip(start, lens)], page)
    cache = _cache(pages, hkv, dim, page, fmt)
    qo, status = torch.empty_like(q).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    params = fastav.make_rotate_params(q=qd, k=kd, v=vd, q_out=qo, pos=pos, frequencies=freq, axis=axis, interleaved=interleaved, norm_eps=1e-5, batch=len(lens))
    fastav.fastav_rotate_write(params, cache, qd, kd, vd, pos.cuda(), _cu(lens).cuda(), table.cuda(), _cuda(torch.tensor(start, dtype=torch.int32)) if any(start) else None,
                               qo, *map(_cuda, norms), status)
    assert int(status) == 0
    _near(qo, *want[0])
    cu = _cu(lens).tolist()
    _check_rows(cache, fmt, table, page, [(b, start[b], [x[cu[b]:cu[b + 1]] for x in want[1]], v[cu[b]:cu[b + 1]]) for b in range(len(lens)) if lens[b]])
    # without queries the cache gets the same
    again = _cache(pages, hkv, dim, page, fmt)
    params = fastav.make_rotate_params(k=kd, v=vd, pos=pos, frequencies=freq, axis=axis, interleaved=interleaved, norm_eps=1e-5, batch=len(lens))
    fastav.fastav_rotate_write(params, again, None, kd, vd, pos.cuda(), _cu(lens).cuda(), table.cuda(), torch.tensor(start, dtype=torch.int32).cuda(), None, None,
                               _cuda(norms[1]), status)
    for a, b in ((cache.k, again.k), (cache.v, again.v)):
        assert torch.equal(a.view(torch.int8), b.view(torch.int8))
    assert torch.equal(cache.k_scale, again.k_scale) and torch.equal(cache.v_scale, again.v_scale)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("scale", [2.0 ** 120, 2.0 ** -95, 2.0 ** -115, 2.0 ** -125])
def test_rows_of_extreme_sizes_go_into_the_cache(scale, fmt):
    """Row maxima near both ends of fp32's range (with values 2^-8 of them that are still normal), and a row of zeros."""
    gen = torch.Generator().manual_seed(21)
    k, v = ((torch.randn(20, 2, 64, generator=gen).clamp(-4, 4) * scale).to(torch.bfloat16) for _ in "kv")
    k[3] = 0
    v[4, 1] = 0
    pos, freq = _positions(gen, 1, 20), fastav.rotary_frequencies(64)
    table, pages = _tables(gen, [20], 16)
    cache = _cache(pages, 2, 64, 16, fmt)
    kd, vd = k.cuda(), v.cuda()
    fastav.fastav_rotate_write(fastav.make_rotate_params(k=kd, v=vd, pos=pos, frequencies=freq), cache, None, kd, vd, pos.cuda(), _cu([20]).cuda(), table.cuda(), None, None)
    _check_rows(cache, fmt, table, 16, [(0, 0, ref.turned(k, pos, freq), v)])


def test_far_and_negative_positions():
    """Out to the ends of 32 bits: angles that fp32 products would miss by whole turns."""
    pos = torch.tensor([0, 1, -1, 999_983, 2 ** 24 + 1, 123_456_789, 2 ** 31 - 1, -2 ** 31, -77_777], dtype=torch.int32)
    freq = [1.0, 0.1234567890123, math.pi, 5e-324, 1e-300, 1e-12, -0.7, 100.0] + [0.01 * i for i in range(24)]
    x = torch.randn(9, 3, 64, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    y = torch.empty_like(x).cuda()
    fastav.fastav_rotate(fastav.make_rotate_params(q=x, q_out=y, pos=pos, frequencies=freq), x.cuda(), None, pos.cuda(), y, None)
    _near(y, *ref.turned(x, pos, freq))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotated_products_depend_on_distance_only(interleaved):
    """<rotated q at m, rotated k at n> is the same for all m with the same m - n: what the rotation is for.  Off by the roundings of 128 products."""
    gen = torch.Generator().manual_seed(7)
    q, k = (torch.randn(1, 1, 128, generator=gen).to(torch.bfloat16) for _ in "qk")
    m = torch.tensor([5, 1005, 70005], dtype=torch.int32)
    qs, ks = q.expand(3, 1, 128).contiguous().cuda(), k.expand(3, 1, 128).contiguous().cuda()
    outs = []
    for x, pos in ((qs, m), (ks, m - 5)):
        y = torch.empty_like(x)
        params = fastav.make_rotate_params(q=x, q_out=y, pos=pos, frequencies=fastav.rotary_frequencies(128), interleaved=interleaved)
        fastav.fastav_rotate(params, x, None, pos.cuda(), y, None)
        outs.append(y.cpu().double()[:, 0])
    dots, size = (outs[0] * outs[1]).sum(1), float((outs[0].abs() * outs[1].abs()).sum(1).max())
    assert float((dots - dots[0]).abs().max()) <= 2 * 2 * 2.0 ** -8 * size


@pytest.mark.parametrize("scale", [2.0 ** 66, 2.0 ** 100, 2.0 ** -60, 2.0 ** -100])
def test_norm_of_huge_and_tiny_rows(scale):
    """Squares that fp32 cannot hold: the norm of a row does not depend on its size while eps is nothing beside it, and tiny rows are x / sqrt(eps)."""
    x = (torch.randn(4, 2, 128, generator=torch.Generator().manual_seed(8)) * scale).to(torch.bfloat16)
    w = torch.ones(128, dtype=torch.bfloat16)
    y = torch.empty_like(x).cuda()
    fastav.fastav_rotate(fastav.make_rotate_params(q=x, q_out=y, norm_eps=1e-6), x.cuda(), None, None, y, None, w.cuda())
    want, size = ref.turned(x, torch.zeros(1, 4, dtype=torch.int32), [], norm=w, eps=1e-6)
    _near(y, want, size)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("normed", [False, True])
def test_a_row_that_is_not_finite_stays_alone(bad, normed):
    x = torch.randn(20, 3, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    y = x.clone()
    y[7, 1, 100] = bad
    pos, w = torch.arange(20, dtype=torch.int32), torch.ones(128, dtype=torch.bfloat16).cuda() if normed else None
    table, cu = torch.tensor([[1, 0]], dtype=torch.int32).cuda(), _cu([20]).cuda()
    got = []
    for rows in (x, y):
        out, k = torch.empty_like(x).cuda(), rows.cuda()
        cache = _cache(2, 3, 128, 16, "fp8")
        params = fastav.make_rotate_params(q=k, k=k, v=k, q_out=out, pos=pos, frequencies=fastav.rotary_frequencies(128))
        fastav.fastav_rotate_write(params, cache, k, k, k, pos.cuda(), cu, table, None, out, w, w)
        ko, vo = torch.empty_like(k), torch.empty_like(k)
        fastav.fastav_cache_read(fastav.make_params(batch=1, total_tokens=20, max_seqlen=20, total_q=0, max_qlen=0, total_keep=0, max_keep=0, num_q_heads=3,
                                                    num_kv_heads=3, head_dim=128, hidden=0, k_out=ko, v_out=vo), cache, table, None, cu, ko, vo)
        assert not torch.isnan(cache.k.float()).any()
        got.append([t.cpu() for t in (out, ko, vo)])
    for clean, dirty in zip(*got):
        rest = torch.ones(20, 3, dtype=torch.bool)
        rest[7, 1] = False
        assert torch.equal(clean[rest], dirty[rest])
    assert bool(torch.isnan(got[1][1][7, 1]).all()) and bool(torch.isnan(got[1][2][7, 1]).all())
    lost = ~torch.isfinite(got[1][0][7, 1])
    assert bool(lost.all()) if normed and not math.isinf(bad) else bool(lost[100]) and bool(lost[36])


def test_rows_without_a_place_and_rows_behind_the_last_sequence():
    n, heads, dim, page = 40, 2, 64, 16
    x = torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    pos, status = torch.arange(n, dtype=torch.int32), torch.zeros(1, dtype=torch.int32, device="cuda")
    params = fastav.make_rotate_params(q=x, k=x, v=x, q_out=x, pos=pos, frequencies=fastav.rotary_frequencies(64), batch=2)

    def write(table, start, lens):
        cache = _cache(3, heads, dim, page, "int8")
        out = torch.full_like(x, 3.0)
        status.zero_()
        fastav.fastav_rotate_write(params, cache, x, x, x, pos.cuda(), _cu(lens).cuda(), torch.tensor(table, dtype=torch.int32).cuda(),
                                   None if start is None else torch.tensor(start, dtype=torch.int32).cuda(), out, device_status=status)
        return cache, out, int(status)

    cache, out, bits = write([[0, 99], [1, -1]], None, [20, 20])
    assert bits == fastav.FASTAV_DEV_BAD_INDEX and bool((cache.k[2] == POISON).all()) and not bool((cache.k[:2] == POISON).all(-1).any())
    assert not bool((out == 3).all(-1).any())                                      # queries do not need a place
    for start in ([20, 0], [-1, 0], [2 ** 31 - 1, 0]):
        assert write([[0, 1], [1, 2]], start, [20, 20])[2] == fastav.FASTAV_DEV_SHAPE_MISMATCH
    cache, out, bits = write([[0, 1], [2, 2]], None, [7, 9])                         # a padded batch
    assert bits == 0 and bool((out[16:] == 3).all()) and not bool((out[:16] == 3).all(-1).any())
    assert bool((cache.k[1] == POISON).all()) and bool((cache.k[0, :, 7:] == POISON).all()) and bool((cache.k[2, :, 9:] == POISON).all())
    cache, out, bits = write([[0, 1], [2, 2]], None, [30, 30])                       # more rows than the host said
    assert bits & fastav.FASTAV_DEV_SHAPE_MISMATCH


def test_offsets_beyond_32_bits():
    heads, dim, page = 8, 128, 256
    pages = (5 << 30) // (heads * dim * page)
    cache = fastav.make_cache(pages, heads, dim, page)
    x = torch.randn(300, heads, dim, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    table, cu = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32).cuda(), _cu([300]).cuda()
    fastav.fastav_rotate_write(fastav.make_rotate_params(k=x, v=x), cache, None, x, x, None, cu, table, None, None)
    codes, scale = cref.quantise(x.cpu(), torch.int8)
    for t in (0, 255, 256, 299):
        at, slot = pages - 1 - t // page, t % page
        assert torch.equal(cache.v[at, :, slot].cpu().double(), codes[t]) and torch.equal(cache.v_scale[at, :, slot].cpu(), scale[t])
    # rows of a projection that lie more than 2^31 elements apart
    far = torch.empty(2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    wide = far.as_strided((3, 1, 128), (2 ** 30, 128, 1))
    wide.copy_(x[:3, :1])
    y = torch.empty(3, 1, 128, dtype=torch.bfloat16, device="cuda")
    fastav.fastav_rotate(fastav.make_rotate_params(q=wide, q_out=y), wide, None, None, y, None)
    assert torch.equal(y, x[:3, :1])


def test_follows_earlier_work_on_a_stream_and_replays():
    """Positions and rows made by kernels right before, on a stream of the caller's; the same call captured and replayed on new contents."""
    n, heads, dim = 2000, 4, 128
    side = torch.cuda.Stream()
    x, y = torch.empty(n, heads, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(n, heads, dim, dtype=torch.bfloat16, device="cuda")
    base, pos = torch.randn(n, heads, dim, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    params = fastav.make_rotate_params(q=x, q_out=y, pos=pos, frequencies=fastav.rotary_frequencies(dim))

    def step(i):
        x.copy_(base + i)
        pos.copy_(torch.arange(n, device="cuda") * (i + 1))
        fastav.fastav_rotate(params, x, None, pos, y, None, stream=torch.cuda.current_stream())

    def check():
        want = ref.turned(x.cpu()[:50], pos.cpu()[:50], fastav.rotary_frequencies(dim))
        _near(y[:50], *want)

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for i in range(4):
            step(i)
            side.synchronize()
            check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(9)
    for add in (1.0, -2.0):
        base.add_(add)
        graph.replay()
        torch.cuda.synchronize()
        check()
