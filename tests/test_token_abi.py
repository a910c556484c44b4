"""Host-side checks of the rotation's, the weighing's and the eviction's entry points that need no GPU: struct layouts, refusals, and the tests' own 64-bit forms."""
import ctypes
import math

import pytest
import torch

import token_reference as ref
from paper_2601_13143_b200 import build as fbuild
from paper_2601_13143_b200 import fastav
from test_cache_abi import BAD_CACHES, FAKE, INVALID, UNSUPPORTED, WORKSPACE, _attend, _cache

NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fastav.library()


def _rotate(**over):
    p = fastav.fastav_rotate_params()
    p.batch, p.total_tokens, p.num_q_heads, p.num_kv_heads, p.head_dim, p.rotary_dim, p.num_axes, p.norm_eps = 2, 30, 8, 2, 64, 32, 3, 1e-6
    p.pos_stride_tok, p.pos_stride_axis = 1, 30
    for side, heads in (("q", 8), ("qo", 8), ("k", 2), ("ko", 2), ("v", 2)):
        setattr(p, side + "_stride_tok", heads * 64)
        setattr(p, side + "_stride_head", 64)
    for i in range(16):
        p.axis[i], p.frequency[i] = i % 3, 0.5 ** i
    for name, value in over.items():
        if name == "axis_of":
            p.axis[value[0]] = value[1]
        elif name == "frequency_of":
            p.frequency[value[0]] = value[1]
        else:
            setattr(p, name, value)
    return p


def _evict(**over):
    p = fastav.fastav_evict_params(3, 500, 300, 8, 8, 4, 32, 0)
    for name, value in over.items():
        setattr(p, name, value)
    return p


def test_struct_layouts_match_the_header():
    r, e = fastav.fastav_rotate_params, fastav.fastav_evict_params
    assert ctypes.sizeof(r) == 40 + 12 * 8 + 64 + 64 * 8 and r.q_stride_tok.offset == 40 and r.axis.offset == 136 and r.frequency.offset == 200
    assert ctypes.sizeof(e) == 32 and e.flags.offset == 28


BAD_TURNS = [(dict(total_tokens=-1), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(rotary_dim=24), UNSUPPORTED), (dict(rotary_dim=80), INVALID),
             (dict(rotary_dim=-16), INVALID), (dict(num_axes=0), INVALID), (dict(num_axes=5), INVALID), (dict(num_axes=2), INVALID), (dict(axis_of=(15, 3)), INVALID),
             (dict(frequency_of=(3, INF)), INVALID), (dict(frequency_of=(3, NAN)), INVALID), (dict(norm_eps=0.0), INVALID), (dict(norm_eps=NAN), INVALID),
             (dict(q_stride_head=60), INVALID), (dict(k_stride_tok=72), INVALID), (dict(k_stride_head=68, k_stride_tok=136), UNSUPPORTED),
             (dict(qo_stride_tok=104), INVALID)]


@pytest.mark.parametrize("over,status", BAD_TURNS + [(dict(num_q_heads=0), INVALID), (dict(ko_stride_head=68, ko_stride_tok=136), UNSUPPORTED)])
def test_rotate_refuses_bad_shapes(lib, over, status):
    assert lib.fastav_rotate(ctypes.byref(_rotate(**over)), FAKE, FAKE, FAKE, FAKE, FAKE, 2 * FAKE, 2 * FAKE, None) == status


def test_rotate_refuses_bad_arguments(lib):
    def call(p=None, q=FAKE, k=FAKE, pos=FAKE, qo=2 * FAKE, ko=2 * FAKE):
        return lib.fastav_rotate(ctypes.byref(p or _rotate()), q, k, pos, None, None, qo, ko, None)

    assert call(q=None) == INVALID and call(ko=None) == INVALID and call(pos=None) == INVALID and call(pos=FAKE + 2) == UNSUPPORTED
    assert call(q=None, k=None, qo=None, ko=None) == INVALID
    assert call(q=FAKE + 8) == UNSUPPORTED and call(ko=FAKE + 2) == UNSUPPORTED
    assert lib.fastav_rotate(ctypes.byref(_rotate()), FAKE, FAKE, FAKE, FAKE, FAKE + 8, 2 * FAKE, 2 * FAKE, None) == UNSUPPORTED
    assert call(p=_rotate(qo_stride_tok=1024), qo=FAKE) == INVALID          # in place, with other strides
    assert call(p=_rotate(total_tokens=0), q=None, k=None, qo=None, ko=None, pos=None) == fastav.FASTAV_OK
    assert lib.fastav_rotate(None, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, None) == INVALID
    with pytest.raises(fastav.FastavError):
        p = _rotate(rotary_dim=24)
        fastav.fastav_rotate(p, None, None, None, None, None, stream=type("S", (), {"cuda_stream": 0}))


@pytest.mark.parametrize("over,status", BAD_TURNS + [(dict(batch=0), INVALID), (dict(num_kv_heads=4), INVALID), (dict(v_stride_head=60), INVALID),
                                                     (dict(v_stride_head=68, v_stride_tok=136), UNSUPPORTED)])
def test_rotate_write_refuses_bad_shapes(lib, over, status):
    c = _cache()
    assert lib.fastav_rotate_write(ctypes.byref(_rotate(**over)), ctypes.byref(c), *[FAKE] * 8, 4, None, 2 * FAKE, None, None) == status


def test_rotate_write_refuses_bad_arguments(lib):
    def call(p=None, c=None, q=FAKE, k=FAKE, v=FAKE, cu=FAKE, table=FAKE, stride=4, qo=2 * FAKE):
        return lib.fastav_rotate_write(ctypes.byref(p or _rotate()), ctypes.byref(c or _cache()), q, k, v, FAKE, None, None, cu, table, stride, None, qo, None, None)

    assert call(k=None) == INVALID and call(v=None) == INVALID and call(cu=None) == INVALID and call(table=None) == INVALID and call(stride=0) == INVALID
    assert call(q=None) == INVALID and call(qo=None) == INVALID and call(v=FAKE + 8) == UNSUPPORTED and call(qo=FAKE + 8) == UNSUPPORTED
    assert call(p=_rotate(total_tokens=0), q=None, k=None, v=None, qo=None) == fastav.FASTAV_OK
    for over, status in BAD_CACHES:
        assert call(c=_cache(**over)) == status


@pytest.mark.parametrize("over,status", [
    (dict(batch=0), INVALID), (dict(total_q=-1), INVALID), (dict(max_qlen=13), INVALID), (dict(num_q_heads=7), INVALID), (dict(max_kv_len=-1), INVALID),
    (dict(batch=4097), UNSUPPORTED), (dict(q_stride_head=60), INVALID), (dict(q_stride_head=68), UNSUPPORTED), (dict(table_stride=0), INVALID)])
def test_weigh_refuses_bad_shapes(lib, over, status):
    assert lib.fastav_cache_weigh(ctypes.byref(_attend(**over)), ctypes.byref(_cache()), FAKE, 1.0, *[FAKE] * 5, None, None, None) == status


def test_weigh_refuses_bad_arguments(lib):
    def call(p=None, c=None, w=FAKE, decay=1.0, q=FAKE, lse=FAKE, cu=FAKE, table=FAKE, lens=FAKE):
        return lib.fastav_cache_weigh(ctypes.byref(p or _attend()), ctypes.byref(c or _cache()), w, decay, q, lse, cu, table, lens, None, None, None)

    for name in ("w", "q", "lse", "cu", "table", "lens"):
        assert call(**{name: None}) == INVALID, name
    assert call(decay=-0.5) == INVALID and call(decay=NAN) == INVALID and call(decay=INF) == INVALID
    assert call(w=FAKE + 8) == UNSUPPORTED and call(q=FAKE + 8) == UNSUPPORTED
    assert call(p=_attend(max_kv_len=0), table=None) == fastav.FASTAV_OK
    for over, status in BAD_CACHES:
        assert call(c=_cache(**over)) == status


@pytest.mark.parametrize("over,status", [
    (dict(batch=0), INVALID), (dict(max_kv_len=-1), INVALID), (dict(max_keep=-1), INVALID), (dict(first=-1), INVALID), (dict(recent=-1), INVALID),
    (dict(batch=1 << 28), UNSUPPORTED), (dict(max_kv_len=2 ** 31 - 1, first=1), UNSUPPORTED)])
def test_evict_refuses_bad_shapes(lib, over, status):
    p, c, out = _evict(**over), _cache(), ctypes.c_size_t(0)
    assert lib.fastav_evict_workspace_bytes(ctypes.byref(p), ctypes.byref(c), ctypes.byref(out)) == status
    assert lib.fastav_cache_evict(ctypes.byref(p), ctypes.byref(c), *[FAKE] * 4, None, 2 * FAKE, None, FAKE, 1 << 40, None, None) == status


def test_evict_refuses_bad_arguments(lib):
    out = ctypes.c_size_t(0)
    assert lib.fastav_evict_workspace_bytes(ctypes.byref(_evict()), ctypes.byref(_cache()), None) == INVALID
    assert lib.fastav_evict_workspace_bytes(ctypes.byref(_evict()), ctypes.byref(_cache()), ctypes.byref(out)) == 0
    need = out.value
    assert need % 256 == 0 and need >= 3 * 2 * 300 * 4

    def call(p=None, c=None, w=FAKE, table=FAKE, lens=FAKE, counts=FAKE, to=None, lens_out=2 * FAKE, ws=FAKE, size=need):
        return lib.fastav_cache_evict(ctypes.byref(p or _evict()), ctypes.byref(c or _cache()), w, table, lens, counts, to, lens_out, None, ws, size, None, None)

    for name in ("w", "table", "lens", "counts", "lens_out"):
        assert call(**{name: None}) == INVALID, name
    assert call(lens_out=FAKE) == INVALID and call(lens_out=FAKE + 8) == INVALID      # the lengths themselves
    assert call(to=FAKE) == INVALID                                                    # the pages themselves: in place is NULL
    assert call(p=_evict(max_kv_len=513)) == INVALID                                   # more tokens than the table has places
    assert call(p=_evict(out_table_stride=4), to=3 * FAKE) == INVALID
    assert call(w=FAKE + 4) == UNSUPPORTED
    assert call(ws=None) == WORKSPACE and call(ws=FAKE + 16) == WORKSPACE and call(size=need - 1) == WORKSPACE
    for over, status in BAD_CACHES:
        assert call(c=_cache(**over)) == status


def test_python_checks_tensors():
    x = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    pos = torch.zeros(3, 5, dtype=torch.int32)
    p = fastav.make_rotate_params(q=x, k=x[:, :2], q_out=x, k_out=x[:, 2:], pos=pos, frequencies=[1.0] * 16, axis=[i % 3 for i in range(16)], interleaved=True)
    assert (p.total_tokens, p.num_q_heads, p.num_kv_heads, p.head_dim, p.rotary_dim, p.num_axes) == (5, 4, 2, 64, 32, 3)
    assert (p.pos_stride_tok, p.pos_stride_axis, p.k_stride_tok, p.flags) == (1, 5, 256, fastav.FASTAV_ROTATE_INTERLEAVED)
    t = fastav.make_rotate_params(q=x, q_out=x, pos=pos.T.contiguous().T, frequencies=[1.0] * 8)
    assert (t.pos_stride_tok, t.pos_stride_axis, t.num_kv_heads) == (3, 1, 0)
    for bad in (dict(), dict(q=x.float()), dict(q=x, q_out=x[:, :2]), dict(q=x, k=x[:3]), dict(q=x, pos=pos.long()), dict(q=x, pos=pos[:, :3]),
                dict(q=x, frequencies=[1.0] * 65), dict(q=x, v=x)):
        with pytest.raises(ValueError):
            fastav.make_rotate_params(**bad)
    cache = fastav.make_cache(3, 2, 64, 32, device="cpu")
    native, lib = fastav._native(), fastav.library()
    for name, count in (("rotate", 10), ("rotate_write", 16), ("cache_weigh", 14), ("cache_evict", 14)):
        with pytest.raises(TypeError):
            getattr(native, name)(*range(count - 1))
    with pytest.raises(ValueError):
        fastav.fastav_cache_weigh(_attend(), cache, torch.zeros(3, 2, 16), *[None] * 5, stream=type("S", (), {"cuda_stream": 0}))
    with pytest.raises(ValueError):
        fastav.fastav_cache_evict(_evict(), cache, None, torch.zeros(3, 8, dtype=torch.int32), *[None] * 4, stream=type("S", (), {"cuda_stream": 0}))
    with pytest.raises(TypeError):
        fastav.fastav_rotate(_evict(), *[None] * 5, stream=type("S", (), {"cuda_stream": 0}))
    assert lib is fastav.library()


def test_frequencies():
    f = fastav.rotary_frequencies(128, 1e6)
    assert len(f) == 64 and f[0] == 1.0 and abs(f[32] - 1e-3) < 1e-15


# ---- the 64-bit forms themselves -----------------------------------------------------------------------

def test_the_angle_is_exact_modulo_a_turn():
    assert abs(ref.angle(1, 2 * math.pi) - 2 * math.pi) < 1e-15 or abs(ref.angle(1, 2 * math.pi)) < 1e-15
    for n in (1, 7, 1000, -3):
        assert abs(math.remainder(ref.angle(n, 0.37) - n * 0.37, 2 * math.pi)) < 1e-12
    assert abs(ref.angle(10 ** 6, 1.0) - 10 ** 6 % (2 * math.pi)) < 1e-9


def test_survivors_by_hand():
    w = torch.tensor([3.0, 1.0, NAN, 2.0, 2.0, 0.0, 5.0])
    assert ref.survivors(w, 3, 0, 0) == [0, 3, 6] and ref.survivors(w, 4, 0, 1) == [0, 3, 4, 6] and ref.survivors(w, 3, 2, 0) == [0, 1, 6]
    assert ref.survivors(w, 2, 3, 3) == [0, 1] and ref.survivors(w, 6, 0, 0) == [0, 1, 3, 4, 5, 6] and ref.survivors(w, 9, 0, 0) == list(range(7))


def test_weights_by_hand():
    k = torch.tensor([[[1.0]], [[2.0]]], dtype=torch.float64)
    out, _ = ref.weigh(torch.tensor([[4.0], [9.0]]), 0.5, 1, torch.ones(2, 1, 1), k, torch.tensor([[0.0], [-INF]]), [2, 2], 1.0)
    assert torch.allclose(out[:, 0], torch.tensor([2 + math.e, math.e ** 2], dtype=torch.float64))
