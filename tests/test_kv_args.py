"""The paged key/value calls refuse bad sizes before they touch a device (runs without a GPU)."""
import ctypes

import pytest

import paper_2607_04415_amd as g
from paper_2607_04415_amd import kv


@pytest.fixture(scope="module")
def lib():
    if not g.LIB_PATH.exists():
        from paper_2607_04415_amd import _build
        _build.build()
    return g.lib()


def cache(**more):
    c = kv.CacheDesc(dtype=kv.BF16, heads=2, D=64, page_tokens=16, num_pages=10)
    for k, v in more.items():
        setattr(c, k, v)
    return c


def attention(**more):
    a = kv.AttentionDesc(dtype=kv.BF16, heads=4, requests=1, width=4, tokens=1, scale=1.0)
    for k, v in more.items():
        setattr(a, k, v)
    return a


def workspace(lib, c, a):
    n = ctypes.c_uint64()
    st = lib.gorio_kv_workspace(ctypes.byref(c), ctypes.byref(a), ctypes.byref(n))
    return st, n.value


@pytest.mark.parametrize("more,text", [
    (dict(dtype=3), "dtype"), (dict(heads=0), "heads"), (dict(D=0), "D="), (dict(D=60), "D="), (dict(D=264), "D="),
    (dict(page_tokens=0), "page_tokens"), (dict(page_tokens=65537), "page_tokens"), (dict(num_pages=0), "num_pages"),
    (dict(num_pages=1 << 31), "num_pages"), (dict(page_stride=4), "strides"), (dict(key_scale=64), "key_scale")])
def test_cache_refusals(lib, more, text):
    assert workspace(lib, cache(**more), attention())[0] == g.EINVAL
    assert text in lib.gorio_last_error().decode()
    c = cache(**more)
    assert lib.gorio_kv_store(ctypes.byref(c), kv.BF16, None, None, 1, 0, 0, None, None) == g.EINVAL


@pytest.mark.parametrize("more,status,text", [
    (dict(dtype=kv.E4M3), g.EINVAL, "q must be"), (dict(dtype=kv.F16), g.EUNSUPPORTED, "own type"),
    (dict(heads=3), g.EINVAL, "multiple"), (dict(heads=0), g.EINVAL, "multiple"), (dict(width=0), g.EINVAL, "width"),
    (dict(width=1 << 30), g.EINVAL, "width"), (dict(tokens=1 << 31), g.EINVAL, "tokens"),
    (dict(q_stride=7), g.EINVAL, "q_stride"), (dict(cap=-1.0), g.EINVAL, "cap"),
    (dict(cap=float("nan")), g.EINVAL, "cap"), (dict(scale=float("inf")), g.EINVAL, "scale")])
def test_attention_refusals(lib, more, status, text):
    assert workspace(lib, cache(), attention(**more))[0] == status
    assert text in lib.gorio_last_error().decode()


def test_null_arguments(lib):
    c, a = cache(), attention()
    assert lib.gorio_kv_attend(None, ctypes.byref(a), None, 0, None) == g.EINVAL
    assert lib.gorio_kv_attend(ctypes.byref(c), None, None, 0, None) == g.EINVAL
    assert lib.gorio_kv_workspace(ctypes.byref(c), ctypes.byref(a), None) == g.EINVAL
    assert lib.gorio_kv_plan(None, None, 1, 16, None, 0, None, 1, 1, None, None, None, None, None, None) == g.EINVAL
    assert lib.gorio_kv_attach(None, 1, 1, None, None, 1, 16, 4, 4, None, None, None, None, None) == g.EINVAL
    assert lib.gorio_kv_store(ctypes.byref(c), kv.BF16, None, None, 1, 0, 0, None, None) == g.EINVAL


def test_sizes_of_zero_are_no_ops(lib):
    c, a = cache(), attention(tokens=0)
    assert lib.gorio_kv_attend(ctypes.byref(c), ctypes.byref(a), None, 0, None) == g.OK
    assert lib.gorio_kv_store(ctypes.byref(c), kv.BF16, None, None, 0, 0, 0, None, None) == g.OK
    assert lib.gorio_kv_plan(None, None, 0, 16, None, 0, None, 1, 1, None, None, None, None, None, None) == g.OK
    assert lib.gorio_kv_attach(None, 0, 1, None, None, 1, 16, 4, 4, None, None, None, None, None) == g.OK


def test_attach_and_plan_refusals(lib):
    assert lib.gorio_kv_attach(None, 1, 0, None, None, 1, 16, 4, 4, None, None, None, None, None) == g.EINVAL
    assert lib.gorio_kv_attach(None, 1, 1025, None, None, 1, 16, 4, 4, None, None, None, None, None) == g.EINVAL
    assert lib.gorio_kv_attach(None, 1, 1, None, None, 1, 0, 4, 4, None, None, None, None, None) == g.EINVAL
    assert lib.gorio_kv_attach(None, 1, 1, None, None, 1, 16, 4, 5, None, None, None, None, None) == g.EINVAL
    assert lib.gorio_kv_plan(None, None, 1, 16, None, 0, None, 0, 1, None, None, None, None, None, None) == g.EINVAL
    assert lib.gorio_kv_plan(None, None, 1 << 31, 16, None, 0, None, 1, 1, None, None, None, None, None, None) == g.EINVAL


@pytest.mark.parametrize("more,text", [(dict(cap=2e38), "cap"), (dict(scale=2e38), "scale"), (dict(scale=-2e38), "scale")])
def test_sizes_past_float32_in_log2_are_refused(lib, more, text):
    assert workspace(lib, cache(), attention(**more))[0] == g.EINVAL
    assert text in lib.gorio_last_error().decode()


def test_rows_that_share_memory_are_refused():
    """Strides of 0 mean packed rows to the library, which would read past an expanded tensor."""
    torch = pytest.importorskip("torch")
    one = torch.zeros(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="share memory"):
        g.KVCache(one.expand(10, 2, 16, 64), one.expand(10, 2, 16, 64))
    with pytest.raises(ValueError, match="share memory"):
        g.KVCache(torch.zeros(10, 1, 16, 64).bfloat16().expand(10, 2, 16, 64), None)
    c = object.__new__(g.KVCache)               # what _rows needs of a cache, without a device
    c.device, c.D, c._layouts, c._codes = one.device, 64, {}, {torch.bfloat16: kv.BF16}
    with pytest.raises(ValueError, match="share memory"):
        c._rows("q", torch.zeros(1, 4, 64).bfloat16().expand(3, 4, 64))
    with pytest.raises(ValueError, match="share memory"):
        c._rows("out", torch.zeros(1024).bfloat16().as_strided((3, 4, 64), (128, 64, 1)))
    wide = torch.zeros(3, 6, 64).bfloat16()
    assert c._rows("q", wide[:, :4]) == (kv.BF16, 6 * 64)
    assert c._rows("q", wide[:1, :4]) == (kv.BF16, 4 * 64)
    assert c._rows("q", wide[:1].expand(1, 6, 64)) == (kv.BF16, 6 * 64)


@pytest.mark.parametrize("kv_heads,group", [(8, 1), (8, 4), (1, 16), (1, 17), (2, 20)])
def test_one_form_is_launched_whatever_rows_are_padding(lib, kv_heads, group):
    """Rows of q may outnumber requests * max_new: over long texts every call needs room for cut tiles."""
    for T in (1, 2, 7, 8, 64, 100, 5000):
        for R in (1, 3, 60, 64, 700):
            for most in (0, 1, 2, 16, 17, 400):
                status, n = workspace(lib, cache(heads=kv_heads, D=128), attention(
                    heads=kv_heads * group, requests=R, tokens=T, max_new=most, width=4096))
                assert status == g.OK and n > 0, (T, R, most)


def test_gradients_are_refused_not_dropped(lib):
    torch = pytest.importorskip("torch")
    pages = torch.zeros(10, 2, 16, 64).bfloat16()
    c = object.__new__(g.KVCache)               # refused before anything that needs a device
    c.device, c.D, c.heads, c._layouts, c._codes = pages.device, 64, 2, {}, {torch.bfloat16: kv.BF16}
    c.keys, c.values, c.key_scale, c.value_scale = pages, pages.clone(), None, None
    rows = torch.zeros(3, 2, 64).bfloat16()
    wants = rows.clone().requires_grad_()
    slopes = torch.zeros(2, requires_grad=True)
    ints = [torch.zeros(shape, dtype=torch.int32) for shape in ((2,), (1,), (1, 4))]
    for call in (lambda: c.attend(wants, *ints), lambda: c.attend(rows, *ints, slopes=slopes),
                 lambda: c.store(wants, rows, None), lambda: c.store(rows, wants, None)):
        with pytest.raises(ValueError, match="no gradients"):
            call()
    c.values.requires_grad_()
    with pytest.raises(ValueError, match="no gradients"):
        c.attend(rows, *ints)
    with torch.no_grad(), pytest.raises(TypeError, match="slots"):
        c.store(wants, rows, torch.zeros(3))
