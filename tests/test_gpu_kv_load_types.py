"""KVCache.load: the type of rows that are given, keys or values, is that of both."""
import pytest

import paper_2607_04415_amd as g
from test_gpu_kv_mx import small

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("side", ["keys", "values"])
def test_rows_given_say_the_type(torch, type, side):
    cache = small(torch, "mx4", 3, "bf16", 4, 2, 64, 16, [3], [40], poison=False)["cache"]
    dtype = torch.bfloat16 if type == "bf16" else torch.float16
    slots = torch.arange(20, device="cuda")
    want = cache.load(slots, dtype)
    rows = torch.zeros(20, 2, 64, dtype=dtype, device="cuda")
    got = cache.load(slots, **{side: rows})
    assert got[side == "values"] is rows
    for x, y in zip(got, want):
        assert x.dtype == dtype and torch.equal(x, y)
