"""Groups of requests whose tables begin alike, against a plain form."""
import numpy as np
import pytest

import paper_2607_04415_amd as g
from test_gpu_kv import ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def share(tables, fills, held, page, least):
    """(first, shared, common), one request at a time."""
    B, width = tables.shape
    common, first, shared = np.zeros(B, int), [], np.zeros(B, int)
    for b in range(B):
        if b:
            n = 0
            while n < width and tables[b, n] == tables[b - 1, n] and (fills is None or fills[b, n] == fills[b - 1, n]):
                n += 1
            common[b] = max(0, min(n, held[b] // page, held[b - 1] // page)) * page
        if b == 0 or common[b] < max(least, 1):
            first.append(b)
    for lo, hi in zip(first, first[1:] + [B]):
        shared[lo:hi] = common[lo + 1:hi].min() if hi - lo > 1 else 0
    return np.array(first + [B] * (B + 1 - len(first))), shared, common


def inputs(rng, B, width, page, groups, fills):
    tables = rng.integers(0, 2**31 - 1, (B, width))
    of = np.sort(rng.integers(0, groups, B))
    for x in range(groups):
        at = np.nonzero(of == x)[0]
        n = rng.integers(0, width + 1)
        if len(at):
            tables[at, :n] = tables[at[0], :n]
    tables[rng.random(B) < 0.1] = -1
    held = rng.integers(0, (width + 2) * page, B)
    held[rng.random(B) < 0.7] = 2**31 - 1
    held[rng.random(B) < 0.05] = -7
    f = np.full((B, width), page) if fills else None
    if fills:
        f[rng.random(f.shape) < 0.002] = 1
    return tables, f, held


@pytest.mark.parametrize("B,width,page,groups,least", [
    (1, 1, 1, 1, 0), (2, 1, 16, 1, 1), (7, 40, 16, 2, 100), (64, 1060, 16, 5, 128), (100, 1024, 1, 3, 1),
    (300, 1025, 24, 30, 5000), (1023, 9, 8, 40, 1), (1024, 9, 8, 1, 1), (1025, 9, 8, 1, 1), (2500, 70, 64, 3, 64),
    (5000, 3, 65536, 5000, 0), (3000, 5, 16, 2, 2**31 - 1)])
@pytest.mark.parametrize("fills", [False, True])
def test_share(torch, B, width, page, groups, least, fills):
    rng = np.random.default_rng([B, width])
    tables, f, held = inputs(rng, B, width, page, groups, fills)
    if groups == 1:                                         # one group over several chunks
        tables[:], held[:] = tables[0], 2**31 - 1
    want = share(tables, f, held, page, least)
    got = g.kv_share(ints(torch, tables), ints(torch, held), page, fills=None if f is None else ints(torch, f), least=least)
    for x, y in zip(got, want):
        assert np.array_equal(x.cpu().numpy(), y)


def test_share_in_a_graph(torch):
    rng = np.random.default_rng(3)
    sets = [inputs(rng, 200, 50, 16, 9, True) for _ in range(4)]
    tables, f, held = (ints(torch, x) for x in sets[0])
    g.kv_share(tables, held, 16, fills=f, least=32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = g.kv_share(tables, held, 16, fills=f, least=32)
    for s in sets:
        for x, y in zip((tables, f, held), s):
            x.copy_(ints(torch, y))
        for x in got:
            x.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, share(s[0], s[1], s[2], 16, 32)):
            assert np.array_equal(x.cpu().numpy(), y)


def test_nothing_to_share_and_refusals(torch):
    none = ints(torch, np.zeros((0, 5)))
    got = g.kv_share(none, ints(torch, []), 16)
    assert got.first.tolist() == [0] and got.shared.numel() == 0
    tables, held = ints(torch, np.zeros((3, 5))), ints(torch, [50, 50, 50])
    with pytest.raises(ValueError, match="held"):
        g.kv_share(tables, held[:2], 16)
    with pytest.raises(ValueError, match="fills"):
        g.kv_share(tables, held, 16, fills=tables[:, :4].contiguous())
    with pytest.raises(TypeError, match="tables"):
        g.kv_share(tables.long(), held, 16)
    with pytest.raises(g.GorioError, match="page_tokens"):
        g.kv_share(tables, held, 0)
    L, x = g.lib(), ints(torch, np.zeros(100))
    at = lambda i: x.data_ptr() + 4 * i
    call = lambda held, common, first, shared: L.gorio_kv_share(at(0), None, held, 3, 5, 16, 1, common, first, shared, None)
    assert call(at(20), at(30), at(40), at(50)) == g.OK
    for bad in ((at(20), at(22), at(40), at(50)), (at(20), at(30), at(32), at(50)), (at(20), at(30), at(40), at(43)),
                (at(20), at(14), at(40), at(50))):
        assert call(*bad) == g.EINVAL and b"overlap" in L.gorio_last_error()
    torch.cuda.synchronize()
