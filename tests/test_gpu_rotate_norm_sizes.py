"""The norm per head near the ends of fp32's range, against the definition in 64 bits (tolerances: those of the rotation's other tests)."""
import math

import pytest
import torch

import token_reference as ref
from paper_2601_13143_b200 import fastav
from test_gpu_cache import _cache, _cu, _tables
from test_gpu_rotate import _check_rows, _near, _positions

pytestmark = pytest.mark.gpu
LARGEST = torch.finfo(torch.float32).max


def _rows(n, heads, dim, scale, seed=8):
    """Normal values, at most 3.9 times `scale` (2^126 of it is below bf16's largest)."""
    return (torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(seed)).clamp(-3.9, 3.9).double() * scale).to(torch.bfloat16)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scale", [2.0 ** 120, 2.0 ** 124, 2.0 ** 125, 2.0 ** 126])
def test_rows_whose_norm_leaves_fp32(scale, dim):
    """The root of the sum of squares itself may be larger than fp32's largest number, not only the squares."""
    x, w = _rows(5, 3, dim, scale), (1 + torch.arange(dim) / dim).to(torch.bfloat16)
    x[2, 1, 5:] = 0                                   # a few large elements, and
    x[3, 2] *= 2.0 ** -110                            # a row of ordinary size between the large ones
    x[4, 0, 7::2] *= 2.0 ** -120                      # elements that are nothing beside their row's others, down to 2^-130 of them
    y = torch.empty_like(x).cuda()
    fastav.fastav_rotate(fastav.make_rotate_params(q=x, q_out=y, norm_eps=1e-6), x.cuda(), None, None, y, None, w.cuda())
    want, size = ref.turned(x, torch.zeros(1, 5, dtype=torch.int32), [], norm=w, eps=1e-6)
    _near(y, want, size)


@pytest.mark.parametrize("scale,eps", [(2.0 ** 63, 2.0 ** 126), (2.0 ** 62, 2.0 ** 127), (2.0 ** 70, 2.0 ** 127), (2.0 ** 40, 2.0 ** 100), (2.0 ** 60, LARGEST)])
def test_eps_counts_beside_squares_of_its_size(scale, eps):
    x, w = _rows(5, 3, 128, scale), torch.ones(128, dtype=torch.bfloat16)
    y = torch.empty_like(x).cuda()
    fastav.fastav_rotate(fastav.make_rotate_params(q=x, q_out=y, norm_eps=eps), x.cuda(), None, None, y, None, w.cuda())
    want, size = ref.turned(x, torch.zeros(1, 5, dtype=torch.int32), [], norm=w, eps=eps)
    _near(y, want, size)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_large_rows_normed_into_the_cache(fmt):
    k, v, w = _rows(20, 2, 128, 2.0 ** 125), _rows(20, 2, 128, 1.0, 9), (1 + torch.arange(128) / 128).to(torch.bfloat16)
    gen = torch.Generator().manual_seed(21)
    pos, freq = _positions(gen, 1, 20), fastav.rotary_frequencies(128)
    table, pages = _tables(gen, [20], 16)
    cache = _cache(pages, 2, 128, 16, fmt)
    kd, vd = k.cuda(), v.cuda()
    params = fastav.make_rotate_params(k=kd, v=vd, pos=pos, frequencies=freq, norm_eps=1e-6)
    fastav.fastav_rotate_write(params, cache, None, kd, vd, pos.cuda(), _cu([20]).cuda(), table.cuda(), None, None, None, w.cuda())
    _check_rows(cache, fmt, table, 16, [(0, 0, ref.turned(k, pos, freq, norm=w, eps=1e-6), v)])


@pytest.mark.parametrize("scale,weight,eps", [(2.0 ** 60, 2.0 ** -100, 1e-6), (2.0 ** 100, 2.0 ** -120, 1e-6), (2.0 ** -40, 2.0 ** 120, 1e-20), (2.0 ** -30, 2.0 ** 100, 1e-20)])
def test_norm_weights_far_from_one(scale, weight, eps):
    """x w / rms is an ordinary number where w / rms is none of fp32's."""
    x, w = _rows(5, 3, 128, scale), ((1 + torch.arange(128) / 128).double() * weight).to(torch.bfloat16)
    y = torch.empty_like(x).cuda()
    fastav.fastav_rotate(fastav.make_rotate_params(q=x, q_out=y, norm_eps=eps), x.cuda(), None, None, y, None, w.cuda())
    want, size = ref.turned(x, torch.zeros(1, 5, dtype=torch.int32), [], norm=w, eps=eps)
    _near(y, want, size)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_a_key_that_leaves_fp32_when_it_is_rotated_is_a_row_that_is_not_finite(fmt):
    """A pair (a, -a) by an eighth of a turn: a sqrt(2) beyond fp32's largest number.  The rows beside it are not touched by it."""
    k, v = _rows(3, 2, 64, 1.0), _rows(3, 2, 64, 1.0, 9)
    k[1, 0, 3], k[1, 0, 35] = 3e38, -3e38
    pos, freq = torch.ones(1, 3, dtype=torch.int32), [math.pi / 4] * 32
    table, pages = _tables(torch.Generator().manual_seed(1), [3], 16)
    cache = _cache(pages, 2, 64, 16, fmt)
    kd, vd = k.cuda(), v.cuda()
    fastav.fastav_rotate_write(fastav.make_rotate_params(k=kd, v=vd, pos=pos, frequencies=freq), cache, None, kd, vd, pos.cuda(), _cu([3]).cuda(), table.cuda(), None, None)
    page = int(table[0, 0])
    assert bool(torch.isnan(cache.k_scale[page, 0, 1])) and not bool(cache.k[page, 0, 1].view(torch.int8).any())
    cache.k_scale[page, 0, 1] = 0
    k[1, 0] = 0
    _check_rows(cache, fmt, table, 16, [(0, 0, ref.turned(k, pos, freq), v)])
