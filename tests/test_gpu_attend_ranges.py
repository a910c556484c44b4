"""fastav_attend where queries, keys or values differ very much in size, for each of its kernels.  Tolerances as derived in test_gpu_attend.py."""
import pytest
import torch

from attend_shapes import GROUP, ROWS, along, direction, long_problem, place, set_queries
from test_gpu_attend import Problem

pytestmark = pytest.mark.gpu


def _normal(p, n, seed=7):
    return torch.randn(n, p.hkv, p.dim, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("bits", [24, 36, 44])
@pytest.mark.parametrize("block", [32, 128])
def test_large_values_that_lose_their_weight(rows, bits, block, fmt):
    """Blocks of keys in turn: values of 1 with logits of 0, then values of 2^-bits with logits of 90 (base 2), which have all the weight."""
    p = long_problem(rows, fmt, n=9000 if rows == 1 else 6000, causal=False)
    n = p.lens[0]
    late = torch.arange(n) // block % 2 == 1
    set_queries(p, direction(p.dim))
    place(p, 0, along(torch.where(late, 90.0, 0.0) + torch.rand(n, generator=p.gen), p.dim)[:, None].expand(-1, p.hkv, -1),
          _normal(p, n) * torch.where(late, 2.0 ** -bits, 1.0)[:, None, None])
    p.run()
    p.check()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("bits", [24, 32, 44])
def test_a_small_value_with_all_the_weight_among_large_ones(rows, bits, fmt):
    """Of sixteen neighbours one has all the weight, and values of 2^-bits of the others'."""
    p = long_problem(rows, fmt, n=1500, causal=False)
    n = p.lens[0]
    heavy = torch.arange(n) % 16 == 5
    set_queries(p, direction(p.dim))
    place(p, 0, along(torch.where(heavy, 80.0, 0.0) + torch.rand(n, generator=p.gen), p.dim)[:, None].expand(-1, p.hkv, -1),
          _normal(p, n) * torch.where(heavy, 2.0 ** -bits, 1.0)[:, None, None])
    p.run()
    p.check()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("rows", ROWS[1:])
@pytest.mark.parametrize("size", [2.0 ** 24, 2.0 ** 40, 1e30])
def test_hidden_keys_with_large_values_do_not_matter(rows, size, fmt):
    """Values of the keys that a causal row does not see are larger by `size`; the last row sees them."""
    p = Problem(8 * GROUP, 8, 128, fmt, 64, [700, rows + 3], [rows, rows], seed=3)
    for b, n in enumerate(p.lens):
        v = _normal(p, n)
        v[n - rows + 1:] *= size
        place(p, b, v=v)
    p.run()
    p.check()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("size", [1e-9, 2.0 ** -60])
def test_groups_of_zero_values_among_small_ones(rows, size, fmt):
    """Every other 16 keys have values of exactly 0, the rest small ones."""
    p = long_problem(rows, fmt, n=2000)
    n = p.lens[0]
    place(p, 0, v=_normal(p, n) * torch.where(torch.arange(n) // 16 % 2 == 0, 0.0, size)[:, None, None])
    p.run()
    p.check()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("exponent", [-60, 100, 116, 120, 122, 124])
def test_values_of_one_extreme_size(rows, exponent, fmt):
    """Up to near the largest bf16: scales of up to 2^119 (e4m3) and 2^121 (int8), in parts that several blocks leave."""
    p = long_problem(rows, fmt, n=2500)
    place(p, 0, v=_normal(p, p.lens[0]).clamp(-3.9, 3.9) * 2.0 ** exponent)
    p.run()
    p.check()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("exponent", [-100, -40, 40, 100, 120])
def test_large_keys_with_small_queries_and_the_reverse(rows, exponent, fmt):
    p = long_problem(rows, fmt, n=600)
    n = p.lens[0]
    q = torch.randn(p.total, p.hq, p.dim, generator=torch.Generator().manual_seed(8))
    set_queries(p, q * 2.0 ** -exponent)
    place(p, 0, k=_normal(p, n).clamp(-3.9, 3.9) * 2.0 ** exponent)
    p.run()
    p.check()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("bits", [16, 20, 24])
def test_small_elements_of_a_query_beside_a_large_one_that_no_key_answers(rows, bits, fmt):
    """The largest element of a query row meets zeros in every key; those that count are 2^-bits of it."""
    p = long_problem(rows, fmt, n=600)
    n = p.lens[0]
    q = torch.randn(p.total, p.hq, p.dim, generator=torch.Generator().manual_seed(8)).clamp(-4, 4) * 2.0 ** -bits
    q[..., 3] = 1.5
    set_queries(p, q)
    k = _normal(p, n) * 2.0 ** bits
    k[..., 3] = 0
    place(p, 0, k=k)
    p.run()
    p.check()


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("query", [0.0, 2.0 ** -120])
def test_logits_that_are_almost_nothing(rows, query):
    """Equal weights: a query row of zeros or of tiny values, and a softmax scale that takes their product below fp32's numbers."""
    p = long_problem(rows, n=333, scale=1e-14)
    set_queries(p, torch.full((p.dim,), query))
    p.run()
    p.check()


@pytest.mark.parametrize("rows", ROWS)
def test_values_near_the_largest_bf16_under_a_growing_maximum(rows):
    """Logits that rise by a few bits from key to key: sums run above their maximum for a while, and nothing may pass fp32's range."""
    p = long_problem(rows, n=2000, causal=False)
    n = p.lens[0]
    set_queries(p, direction(p.dim))
    place(p, 0, along(torch.arange(n) % 64 * 0.9, p.dim)[:, None].expand(-1, p.hkv, -1), _normal(p, n).clamp(-1.9, 1.9) * 2.0 ** 126)
    p.run()
    p.check()


@pytest.mark.parametrize("entries", [1999, 2003])
def test_lists_of_more_entries_than_shared_memory_has_room_for(entries):
    """Two rows of 16 heads on one KV head each, head_dim 128: up to 2,000 entries are listed in shared memory."""
    lens, rows = [i % 9 for i in range(entries - 1)], [2] * (entries - 1)
    p = Problem(16, 1, 128, "int8", 16, lens, rows, prefix_lens=[5], groups=[3, 1501], seed=16)
    p.run()
    p.check()


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("some", [False, True])
def test_a_value_is_its_code_times_its_scale_whatever_the_sign(rows, some):
    """Scales that are negative, all of them or every third one; values of a cache that others filled."""
    p = long_problem(rows, n=700)
    t = torch.arange(700)
    to, slot, flip = p.tables[0][0].long()[t // 64], t % 64, torch.where((t % 3 == 0) | (not some), -1.0, 1.0)
    for scales, which in ((p.cache.k_scale, 0), (p.cache.v_scale, 1)):
        scales[to.cuda(), :, slot.cuda()] *= flip[:, None].cuda()
        p.tokens[0][which] *= flip[:, None, None]
    p.run()
    p.check()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("size", [0.0, 2.0 ** -62, 1e-9, 1e9, 2.0 ** 110])
def test_log_sum_exps_near_zero_beside_values_of_any_size(rows, size, fmt):
    """A few keys, logits of a few bits: the log-sum-exp is small and the exponents of the values' scales are not."""
    p = Problem(8 * GROUP, 8, 64, fmt, 64, [1, 2, 3, 5], [rows] * 4, causal=False, seed=17)
    for b, n in enumerate(p.lens):
        place(p, b, v=_normal(p, n, seed=18 + b) * size)
    p.run()
    p.check()
