"""Pages with powers, loads and sharing: bad sizes are refused before a device is touched (runs without a GPU)."""
import ctypes

import pytest

import paper_2607_04415_amd as g
from paper_2607_04415_amd import kv
from test_kv_args import attention, cache, lib, workspace  # noqa: F401


@pytest.mark.parametrize("dtype", [kv.MX8, kv.MX4])
@pytest.mark.parametrize("more,text", [
    (dict(D=40), "multiple of 32"), (dict(D=264), "D="), (dict(page_stride=2 * 16 * 64 + 8, head_stride=1024, token_stride=64), "strides"),
    (dict(page_stride=2048, head_stride=1024, token_stride=72), "strides"), (dict(key_scale=64), "key_scale"),
    (dict(value_scale=64), "value_scale"), (dict(num_pages=0), "num_pages")])
def test_cache_refusals(lib, dtype, more, text):  # noqa: F811
    c = cache(dtype=dtype, **more)
    assert workspace(lib, c, attention())[0] == g.EINVAL
    assert text in lib.gorio_last_error().decode()
    assert lib.gorio_kv_store(ctypes.byref(c), kv.BF16, None, None, 1, 0, 0, None, None) == g.EINVAL
    assert lib.gorio_kv_load(ctypes.byref(c), kv.BF16, None, 1, None, None, 0, 0, None) == g.EINVAL
    assert text in lib.gorio_last_error().decode()


@pytest.mark.parametrize("dtype", [3, 6, 255, 2**32 - 1])
def test_cache_types(lib, dtype):  # noqa: F811
    assert workspace(lib, cache(dtype=dtype), attention())[0] == g.EINVAL
    assert "gorio_kv_dtype" in lib.gorio_last_error().decode()


@pytest.mark.parametrize("dtype", [kv.MX8, kv.MX4])
@pytest.mark.parametrize("q", [kv.BF16, kv.F16])
def test_both_kinds_of_queries_read_them(lib, dtype, q):  # noqa: F811
    assert workspace(lib, cache(dtype=dtype), attention(dtype=q)) == (g.OK, 0)
    assert workspace(lib, cache(dtype=dtype), attention(dtype=dtype))[0] == g.EINVAL
    c = cache(dtype=dtype)
    assert lib.gorio_kv_store(ctypes.byref(c), q, None, None, 0, 0, 0, None, None) == g.OK
    assert lib.gorio_kv_load(ctypes.byref(c), q, None, 0, None, None, 0, 0, None) == g.OK


@pytest.mark.parametrize("of,dtype,tokens,strides,status,text", [
    (kv.BF16, kv.E4M3, 1, (0, 0), g.EINVAL, "bf16 or f16"), (kv.MX4, kv.MX4, 1, (0, 0), g.EINVAL, "bf16 or f16"),
    (kv.BF16, kv.F16, 1, (0, 0), g.EUNSUPPORTED, "own type"), (kv.MX8, kv.F16, 1 << 31, (0, 0), g.EINVAL, "tokens"),
    (kv.MX8, kv.F16, 1, (132, 0), g.EINVAL, "multiples of 8"), (kv.MX8, kv.F16, 1, (0, 132), g.EINVAL, "multiples of 8"),
    (kv.MX8, kv.F16, 2, (120, 0), g.EINVAL, "at least"), (kv.MX8, kv.F16, 2, (0, 64), g.EINVAL, "at least"),
    (kv.MX8, kv.F16, 1, (0, 0), g.EINVAL, "keys is NULL"), (kv.BF16, kv.BF16, 1, (0, 0), g.EINVAL, "keys is NULL")])
def test_load_refusals(lib, of, dtype, tokens, strides, status, text):  # noqa: F811
    c = cache(dtype=of)
    assert lib.gorio_kv_load(ctypes.byref(c), dtype, None, tokens, None, None, *strides, None) == status
    assert text in lib.gorio_last_error().decode()


@pytest.mark.parametrize("requests,width,page,least,text", [
    ((1 << 20) + 1, 4, 16, 1, "requests"), (2**64 - 1, 4, 16, 1, "requests"), (1, 0, 16, 1, "width"),
    (1, 1 << 30, 16, 1, "width"), (1, 4, 0, 1, "page_tokens"), (1, 4, 65537, 1, "page_tokens"),
    (1, 4, 16, 1 << 31, "least"), (1, 4, 16, 1, "tables is NULL")])
def test_share_refusals(lib, requests, width, page, least, text):  # noqa: F811
    assert lib.gorio_kv_share(None, None, None, requests, width, page, least, None, None, None, None) == g.EINVAL
    assert text in lib.gorio_last_error().decode()
    assert lib.gorio_kv_share(None, None, None, 0, 4, 16, 1, None, None, None, None) == g.OK


def test_sharing(lib):  # noqa: F811
    c, a = cache(dtype=kv.MX4), attention(requests=5, tokens=7, width=1 << 20)
    n, s = ctypes.c_uint64(), kv.SharingDesc(groups=2)
    need = lambda share: lib.gorio_kv_workspace_shared(ctypes.byref(c), ctypes.byref(a), share, ctypes.byref(n))
    assert need(ctypes.byref(s)) == g.OK
    assert n.value >= 7 * 4 * (64 + 2) * 4                      # of each row its sums, a maximum and a sum of weights
    for more in (dict(window=10), dict(window=0, width=9000)):  # nothing is shared then, or not worth it
        for k, v in more.items():
            setattr(a, k, v)
        assert need(ctypes.byref(s)) == g.OK and n.value == workspace(lib, c, a)[1]
    assert need(None) == g.EINVAL and b"sharing is NULL" in lib.gorio_last_error()
    for groups in (0, 6, 2**32 - 1):
        s.groups = groups
        assert need(ctypes.byref(s)) == g.EINVAL and b"groups" in lib.gorio_last_error()
        assert lib.gorio_kv_attend_shared(ctypes.byref(c), ctypes.byref(a), ctypes.byref(s), None, 0, None) == g.EINVAL
    s.groups = 5
    assert lib.gorio_kv_attend_shared(ctypes.byref(c), ctypes.byref(a), None, None, 0, None) == g.EINVAL
    assert lib.gorio_kv_attend_shared(ctypes.byref(c), ctypes.byref(a), ctypes.byref(s), None, 0, None) == g.EINVAL
    assert b"q is NULL" in lib.gorio_last_error()
    a.tokens = 0
    assert lib.gorio_kv_attend_shared(ctypes.byref(c), ctypes.byref(a), ctypes.byref(s), None, 0, None) == g.OK
