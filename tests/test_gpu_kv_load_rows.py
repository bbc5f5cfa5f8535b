"""gorio_kv_load into parts of wider rows: parts that meet are refused, parts that alternate are written."""
import pytest

import paper_2607_04415_amd as g

pytestmark = pytest.mark.gpu
T, H, D = 7, 2, 64
ROW = H * D


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def cache(torch):
    gen = torch.Generator().manual_seed(4)
    return g.KVCache(*(torch.randn(3, H, 8, D, generator=gen).bfloat16().cuda() for _ in range(2)))


def parts(torch, keys, values):
    """Rows of one array at (first element, stride) each."""
    flat = torch.full((8 * T * ROW,), 5.0, dtype=torch.bfloat16, device="cuda")
    return flat, *(flat.as_strided((T, H, D), (step, D, 1), at) for at, step in (keys, values))


@pytest.mark.parametrize("keys,values", [
    ((0, 3 * ROW), (0, 3 * ROW)), ((0, 3 * ROW), (ROW - 8, 3 * ROW)), ((ROW - 8, 3 * ROW), (0, 3 * ROW)),
    ((0, 2 * ROW), (2 * ROW, 2 * ROW)), ((0, 2 * ROW), (ROW + 8, 2 * ROW)), ((2 * ROW, 2 * ROW), (0, 2 * ROW)),
    ((0, 2 * ROW), (12 * ROW, 2 * ROW)), ((0, 3 * ROW), (ROW, 2 * ROW)), ((0, ROW), (6 * ROW + 8, 2 * ROW)),
    ((0, ROW + 8), (ROW + 8, ROW + 8)), ((8, ROW + 8), (0, ROW + 8))])
def test_rows_that_meet_are_refused(torch, cache, keys, values):
    flat, k, v = parts(torch, keys, values)
    with pytest.raises(g.GorioError, match="overlap"):
        cache.load(torch.arange(T, device="cuda"), keys=k, values=v)
    torch.cuda.synchronize()
    assert (flat == 5).all()


@pytest.mark.parametrize("keys,values", [
    ((0, 2 * ROW), (ROW, 2 * ROW)), ((ROW, 2 * ROW), (0, 2 * ROW)), ((0, 3 * ROW), (2 * ROW, 3 * ROW)),
    ((0, 3 * ROW + 8), (ROW + 8, 3 * ROW + 8)), ((0, 4 * ROW), (ROW, 2 * ROW)), ((0, 2 * ROW), (13 * ROW, 2 * ROW)),
    ((0, ROW), (7 * ROW, 2 * ROW)), ((20 * ROW, ROW), (0, 3 * ROW))])
def test_rows_that_alternate(torch, cache, keys, values):
    flat, k, v = parts(torch, keys, values)
    slots = torch.arange(T, device="cuda") * 3 % 24
    want = cache.load(slots)
    cache.load(slots, keys=k, values=v)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    assert (flat != 5).sum() <= 2 * T * ROW
