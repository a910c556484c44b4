"""Host-side checks of the cache's and the attention's entry points that need no GPU: struct layouts, workspace sizes, refusals."""
import ctypes

import pytest
import torch

from paper_2601_13143_b200 import build as fbuild
from paper_2601_13143_b200 import fastav

INVALID, UNSUPPORTED, WORKSPACE = fastav.FASTAV_ERR_INVALID_ARG, fastav.FASTAV_ERR_UNSUPPORTED, fastav.FASTAV_ERR_WORKSPACE
FAKE = 0x100000  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fastav.library()


def _cache(**over):
    c = fastav.fastav_cache(0, 64, 10, 2, 64, FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE)
    for name, value in over.items():
        setattr(c, name, value)
    return c


def _params(**over):
    base = dict(batch=2, total_tokens=300, max_seqlen=200, total_q=0, max_qlen=0, total_keep=150, max_keep=100, num_q_heads=8, num_kv_heads=2, head_dim=64,
                hidden=0)
    base.update(over)
    return fastav.make_params(**base)


def _attend(**over):
    p = fastav.fastav_attend_params(3, 12, 8, 8, 500, 8, 0, 0, 0, 0, 8 * 64, 64, 8 * 64, 64, 0.0, fastav.FASTAV_CAUSAL)
    for name, value in over.items():
        setattr(p, name, value)
    return p


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(fastav.fastav_cache) == 56 and fastav.fastav_cache.k.offset == 24                     # 5 int32, padding, 4 pointers
    assert ctypes.sizeof(fastav.fastav_attend_params) == 80 and fastav.fastav_attend_params.q_stride_tok.offset == 40  # 10 int32, 4 int64, float, uint32


BAD_CACHES = [(dict(format=2), UNSUPPORTED), (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=512), UNSUPPORTED),
              (dict(num_pages=0), INVALID), (dict(k=None), INVALID), (dict(v_scale=None), INVALID), (dict(k=FAKE + 64), UNSUPPORTED),
              (dict(k_scale=FAKE + 8), UNSUPPORTED), (dict(num_pages=1 << 24, page_tokens=256), UNSUPPORTED)]


@pytest.mark.parametrize("over,status", BAD_CACHES + [(dict(num_kv_heads=4), INVALID), (dict(head_dim=128), INVALID)])
def test_rows_refuse_a_bad_cache(lib, over, status):
    p, c = _params(), _cache(**over)
    assert lib.fastav_cache_write(ctypes.byref(p), ctypes.byref(c), FAKE, FAKE, FAKE, None, None, FAKE, 4, None, None, None) == status
    assert lib.fastav_cache_read(ctypes.byref(p), ctypes.byref(c), FAKE, 4, None, FAKE, FAKE, FAKE, None, None) == status


def test_rows_refuse_bad_arguments(lib):
    c, p = _cache(), _params()

    def write(p=p, k=FAKE, v=FAKE, cu=FAKE, idx=None, cu_keep=None, table=FAKE, stride=4):
        return lib.fastav_cache_write(ctypes.byref(p), ctypes.byref(c), k, v, cu, idx, cu_keep, table, stride, None, None, None)

    assert write(k=None) == INVALID and write(v=None) == INVALID and write(cu=None) == INVALID and write(table=None) == INVALID and write(stride=0) == INVALID
    assert write(idx=FAKE) == INVALID and write(cu_keep=FAKE) == INVALID       # a list without its bounds, bounds without a list
    assert write(k=FAKE + 8) == UNSUPPORTED
    assert write(p=_params(batch=0)) == INVALID and write(p=_params(max_seqlen=301)) == INVALID
    assert write(p=_params(total_keep=301), idx=FAKE, cu_keep=FAKE) == INVALID
    bad = _params()
    bad.v_stride_head = 60
    assert write(p=bad) == INVALID
    bad.v_stride_head = 68
    assert write(p=bad) == UNSUPPORTED
    assert lib.fastav_cache_write(None, ctypes.byref(c), FAKE, FAKE, FAKE, None, None, FAKE, 4, None, None, None) == INVALID
    assert lib.fastav_cache_write(ctypes.byref(p), None, FAKE, FAKE, FAKE, None, None, FAKE, 4, None, None, None) == INVALID
    assert write(p=_params(total_tokens=0, max_seqlen=0, total_keep=0, max_keep=0), k=None, v=None) == fastav.FASTAV_OK   # nothing to do, nothing enqueued
    bad = _params()
    bad.ko_stride_tok = 64  # two heads do not fit
    assert lib.fastav_cache_read(ctypes.byref(bad), ctypes.byref(c), FAKE, 4, None, FAKE, FAKE, FAKE, None, None) == INVALID


@pytest.mark.parametrize("over,status", [
    (dict(batch=0), INVALID), (dict(total_q=-1), INVALID), (dict(max_qlen=13), INVALID), (dict(num_q_heads=7), INVALID), (dict(max_kv_len=-1), INVALID),
    (dict(num_prefixes=-1), INVALID), (dict(num_prefixes=1, max_prefix_q=13), INVALID), (dict(batch=4097), UNSUPPORTED),
    (dict(batch=4000, num_prefixes=100), UNSUPPORTED), (dict(batch=4096, max_qlen=1 << 20, total_q=1 << 26, max_kv_len=1 << 30), UNSUPPORTED),
])
def test_attend_refuses_bad_shapes(lib, over, status):
    out = ctypes.c_size_t(0)
    p, c = _attend(**over), _cache()
    assert lib.fastav_attend_workspace_bytes(ctypes.byref(p), ctypes.byref(c), ctypes.byref(out)) == status
    assert lib.fastav_attend(ctypes.byref(p), ctypes.byref(c), *[FAKE] * 7, FAKE, None, FAKE, 1 << 40, None, None) == status


@pytest.mark.parametrize("over,status", BAD_CACHES)
def test_attend_refuses_a_bad_cache(lib, over, status):
    out, p, c = ctypes.c_size_t(0), _attend(), _cache(**over)
    assert lib.fastav_attend_workspace_bytes(ctypes.byref(p), ctypes.byref(c), ctypes.byref(out)) == status


def test_attend_refuses_bad_arguments(lib):
    c, out = _cache(), ctypes.c_size_t(0)
    assert lib.fastav_attend_workspace_bytes(ctypes.byref(_attend()), ctypes.byref(c), None) == INVALID
    assert lib.fastav_attend_workspace_bytes(ctypes.byref(_attend()), ctypes.byref(c), ctypes.byref(out)) == 0 and out.value % 256 == 0
    need = out.value

    def call(p=None, q=FAKE, cu=FAKE, table=FAKE, lens=FAKE, prefix=(None, None, None), o=FAKE, ws=FAKE, size=need):
        return lib.fastav_attend(ctypes.byref(p or _attend()), ctypes.byref(c), q, cu, table, lens, *prefix, o, None, ws, size, None, None)

    assert call(q=None) == INVALID and call(cu=None) == INVALID and call(table=None) == INVALID and call(lens=None) == INVALID and call(o=None) == INVALID
    assert call(ws=None) == WORKSPACE and call(ws=FAKE + 16) == WORKSPACE and call(size=need - 1) == WORKSPACE
    assert call(q=FAKE + 8) == UNSUPPORTED and call(o=FAKE + 2) == UNSUPPORTED
    assert call(p=_attend(q_stride_head=60)) == INVALID and call(p=_attend(o_stride_head=68)) == UNSUPPORTED
    with_prefix = _attend(num_prefixes=1, max_prefix_len=100, prefix_table_stride=4, max_prefix_q=12)
    assert lib.fastav_attend_workspace_bytes(ctypes.byref(with_prefix), ctypes.byref(c), ctypes.byref(out)) == 0 and out.value > need
    for missing in range(3):
        prefix = [FAKE] * 3
        prefix[missing] = None
        assert call(p=with_prefix, prefix=prefix, size=1 << 40) == INVALID
    assert call(p=_attend(total_q=0, max_qlen=0), q=None, o=None, size=1 << 40) == fastav.FASTAV_OK


def test_python_handles_check_their_tensors():
    k, s = torch.zeros(4, 2, 16, 64, dtype=torch.int8), torch.zeros(4, 2, 16)
    handle = fastav.KvCache(k, k.clone(), s, s.clone()).struct
    assert (handle.format, handle.page_tokens, handle.num_pages, handle.num_kv_heads, handle.head_dim) == (0, 16, 4, 2, 64)
    for bad in ((k.float(), k, s, s), (k, k[:2], s, s), (k, k, s[:, :1], s), (k, k, s.double(), s), (k.transpose(1, 2), k.transpose(1, 2), s, s)):
        with pytest.raises(ValueError):
            fastav.KvCache(*bad)
    made = fastav.make_cache(3, 2, 64, 32, fastav.FASTAV_CACHE_FP8, device="cpu")
    assert made.k.dtype == torch.float8_e4m3fn and made.k.shape == (3, 2, 32, 64) and made.struct.format == fastav.FASTAV_CACHE_FP8
    with pytest.raises(ValueError):
        fastav._table(torch.zeros(4, 4))
    wide = torch.zeros(4, 10, dtype=torch.int32)
    assert fastav._table(wide[:, 2:6]) == 10 and fastav._table(wide[:1, 2:6]) == 4 and fastav._table(None) == 0


@pytest.mark.parametrize("name,count,numbers", [("cache_write", 13, {9: 4}), ("cache_read", 11, {4: 4}), ("attend", 15, {})])
def test_the_c_module_passes_on_what_it_is_given(lib, name, count, numbers):
    """Marshalling: a wrong number of arguments and a params of another type are refused in Python, a call without tensors by the library."""
    native = fastav._native()
    function = getattr(native, name)
    with pytest.raises(TypeError):
        function(*range(count - 1))
    with pytest.raises(TypeError):
        fastav._struct(_params(), fastav.fastav_attend_params)
    p, c = (_attend() if name == "attend" else _params()), _cache()
    arguments = [ctypes.cast(getattr(lib, "fastav_" + name), ctypes.c_void_p).value, ctypes.addressof(p), ctypes.addressof(c)] + [None] * (count - 4) + [0]
    for at, value in numbers.items():
        arguments[at] = value
    assert function(*arguments) == INVALID
    arguments[3 if name != "cache_read" else 5] = "not a tensor"
    with pytest.raises(AttributeError):
        function(*arguments)
