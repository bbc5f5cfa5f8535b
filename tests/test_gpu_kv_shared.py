"""Attention of a batch whose requests share their first pages: as without sharing, by kv_reference.attend."""
import ctypes

import numpy as np
import pytest

import kv_reference as ref
import mx_reference as mx
import paper_2607_04415_amd as g
from paper_2607_04415_amd import kv
from test_gpu_kv import call, holds, ints, setup
from test_gpu_kv_mx import small

pytestmark = pytest.mark.gpu
NAN = float("nan")
ROOM = 200_000_000         # elements of keys and values that tables have room for, from which groups are computed


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def inputs(torch, seed, type, cache, H, KV, D, page, groups, news, own, shared, *, poison=True, **more):
    """Requests of which each group's first `shared` positions (one number a group) lie in the same pages;
    `own`: how many positions each has behind them.  What no row sees is NaN."""
    of = np.repeat(np.arange(len(groups)), groups)
    shared = np.array(shared)[of] // page * page
    lens = np.array(own) + shared
    # calls whose tables have room for little are computed without groups: these have room for more
    more.setdefault("width", ROOM // (2 * KV * D * page * len(lens)) + 1 + int(lens.max()) // page)
    make = (lambda *a, **k: small(torch, cache, *a, **k)) if cache in mx.KINDS else \
        (lambda seed, type, *a, **k: setup(torch, seed, type, cache, *a, **k))
    a = make(seed, type, H, KV, D, page, news, np.maximum(lens, 0), poison=False, **more)
    first = np.concatenate([[0], np.cumsum(groups)])
    for b in range(len(lens)):
        n, lead = shared[b] // page, first[of[b]]
        a["tables"][b, :n] = a["tables"][lead, :n]
        if a.get("fills") is not None:
            a["fills"][b, :n] = a["fills"][lead, :n]
    a["first"], a["shared"] = first, shared
    if poison:
        c = a["cache"]
        pages = c.keys.shape[0]
        seen = np.zeros((pages, page), bool)
        for b in range(len(lens)):
            for i in range(news[b]):
                j = ref.visible(b, int(lens[b]) - news[b] + i, int(lens[b]), a)
                seen[a["tables"][b, j // page], j % page] = True
        bad = torch.from_numpy(~seen).cuda()
        if cache in mx.KINDS:
            for x in (c.key_scale, c.value_scale):
                x.view(torch.uint8).permute(0, 2, 1, 3)[bad] = 255
        elif cache == "e4m3":
            for x in (c.keys, c.values):
                x.view(torch.uint8).permute(0, 2, 1, 3)[bad] = 127
        else:
            for x in (c.keys, c.values):
                x.permute(0, 2, 1, 3)[bad] = NAN
                x.permute(0, 2, 1, 3)[..., ::2][bad] = float("inf")
    return a


def grouped(a):
    """Whether such a call has room for the sums over shared positions."""
    T, H, D = a["q"].shape
    B, width = a["tables"].shape
    desc = kv.AttentionDesc(dtype=kv.BF16 if a["type"] == "bf16" else kv.F16, heads=H, requests=B, width=width, tokens=T,
                            prefix=None if a.get("prefix") is None else 64, window=a["window"], scale=1.0)
    share, n = kv.SharingDesc(groups=B), [ctypes.c_uint64() for _ in range(2)]
    L, c = g.lib(), a["cache"]._ref
    assert L.gorio_kv_workspace(c, ctypes.byref(desc), ctypes.byref(n[0])) == g.OK
    assert L.gorio_kv_workspace_shared(c, ctypes.byref(desc), ctypes.byref(share), ctypes.byref(n[1])) == g.OK
    return n[0].value != n[1].value


def sharing(torch, a, first=None):
    return g.KVSharing(ints(torch, a["first"] if first is None else first), ints(torch, a["shared"]))


def check(torch, a, want=None, **more):
    want = ref.attend(a) if want is None else want
    holds(torch, a, call(torch, a, sharing=sharing(torch, a), **more), want)
    assert grouped(a) == (not a["window"] or a.get("prefix") is not None)
    return want


KINDS = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "mx8"), ("bf16", "mx4")]


@pytest.mark.parametrize("type,cache", KINDS)
@pytest.mark.parametrize("H,KV,D,page", [(4, 4, 64, 16), (8, 2, 128, 16), (6, 1, 96, 24), (10, 2, 160, 48), (4, 2, 256, 7),
                                         (40, 1, 32, 1)])
def test_shapes(torch, type, cache, H, KV, D, page):
    """Groups of one, two and four requests, one without anything new, one that shares too little for a block."""
    a = inputs(torch, D + page, type, cache, H, KV, D, page, [1, 2, 4, 2], [1, 1, 5, 1, 0, 33, 2, 1, 1],
               [1, 5, 9, 130, 70, 64, 3, 20, 1], [130, 200, 336, 50])
    want = check(torch, a)
    check(torch, a, want, max_new=33)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3"), ("bf16", "mx4")])
@pytest.mark.parametrize("news", [[1, 1, 1, 1, 1], [3, 1, 0, 4, 1], [40, 1, 70, 2, 9]])
@pytest.mark.parametrize("opts", [
    dict(cap=20.0), dict(cap=0.5), dict(cap=300.0), dict(slopes=True), dict(slopes=True, cap=30.0), dict(window=100),
    dict(window=100, prefix=[250, 30, 0, 400, 2**31 - 1]), dict(window=3, prefix=[0, 0, 0, 0, 0]), dict(fills=True),
    dict(fills=True, prefix=[256, 256, 100, -3, 192], slopes=True), dict(absent=0.5), dict(absent=1.0),
    dict(fills=True, absent=0.3, prefix=[2**31 - 1, 64, 256, 0, 500], slopes=True, cap=40.0, window=90),
    dict(scale=-0.3), dict(scale=0.0), dict(scale=0.0, slopes=True), dict(scale=-0.2, slopes=True)])
def test_masks(torch, type, cache, news, opts):
    """What a row sees of the shared positions goes by its own position, prefix, window and length."""
    a = inputs(torch, 3, type, cache, 4, 2, 64, 16, [3, 2], news, [80, 90, 71, 75, 130], [256, 192], **opts)
    check(torch, a, max_new=max(news))


@pytest.mark.parametrize("cache", ["bf16", "mx8"])
@pytest.mark.parametrize("D", [64, 128, 200])
def test_shared_positions_that_not_all_rows_see(torch, cache, D):
    """Chunks inside what is shared, and a request that ends in it: neither sees what is behind its rows."""
    D = D if cache == "bf16" else D // 32 * 32
    a = inputs(torch, D, "bf16", cache, 4, 2, D, 16, [3, 2], [50, 1, 20, 90, 7], [3, -60, -100, 40, -200], [256, 304])
    check(torch, a)
    a = inputs(torch, D, "bf16", cache, 4, 2, D, 16, [3, 2], [50, 1, 20, 90, 7], [3, -60, -100, 40, -200], [256, 304],
               prefix=[200, 196, 10, 304, 104], fills=True)
    check(torch, a)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "mx8"), ("bf16", "mx4"), ("bf16", "e4m3")])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_long(torch, type, cache, D):
    """Shared positions divided among workgroups; own ones too, and rows of both forms."""
    a = inputs(torch, D, type, cache, 4, 2, D, 16, [4, 2], [1, 1, 30, 1, 2, 1], [9, 2100, 90, 1, 700, 64], [2600, 1500],
               fills=True, prefix=[2600, 2600, 2592, 2601, 1500, 1000], poison=False)
    check(torch, a, max_new=30)


@pytest.mark.parametrize("groups,news", [([1300], 1), ([2] * 700, 1), ([1] * 300 + [900, 3], 1), ([40, 300], 3)])
def test_many_requests(torch, groups, news):
    """More requests to a group, and more groups, than a workgroup has threads; several tiles to a group."""
    rng = np.random.default_rng(len(groups))
    B = sum(groups)
    n = rng.integers(0, news + 1, B) if news > 1 else np.ones(B, int)
    a = inputs(torch, B, "bf16", "bf16", 2, 1, 64, 16, groups, n.tolist(), np.maximum(n, rng.integers(1, 40, B)),
               [64 + 16 * (i % 9) for i in range(len(groups))], poison=False)
    check(torch, a)


def test_groups_as_found(torch):
    """kv_share's own answer, with its empty groups; and one group a request, which shares nothing or all alone."""
    a = inputs(torch, 5, "bf16", "bf16", 8, 2, 128, 16, [3, 1, 2], [1, 4, 1, 1, 1, 30], [40, 50, 20, 9, 8, 77],
               [320, 100, 640], poison=False)
    want = ref.attend(a)
    held = np.array(a["lens"]) - np.array([1, 4, 1, 1, 1, 30])
    got = g.kv_share(ints(torch, a["tables"]), ints(torch, held), 16, least=64)
    assert got.first.tolist() == [0, 3, 4, 6, 6, 6, 6] and got.shared.tolist() == [320, 320, 320, 0, 640, 640]
    holds(torch, a, call(torch, a, sharing=got), want)
    assert grouped(a)
    holds(torch, a, call(torch, a, sharing=got, max_new=30), want)
    alone = g.KVSharing(ints(torch, np.arange(7)), ints(torch, a["shared"]))
    holds(torch, a, call(torch, a, sharing=alone), want)
    nothing = g.KVSharing(ints(torch, [0, 6]), ints(torch, np.zeros(6)))
    holds(torch, a, call(torch, a, sharing=nothing), want)
    padded = g.KVSharing(ints(torch, [0, 3, 3, 4, 6]), ints(torch, a["shared"]))      # an empty group between
    holds(torch, a, call(torch, a, sharing=padded), want)


def test_values_out_of_range_stay_inside(torch):
    """first and shared that make no sense: rows may be wrong, and no memory but the call's is touched."""
    a = inputs(torch, 6, "bf16", "bf16", 4, 2, 64, 16, [3, 2], [1, 1, 2, 1, 30], [40, 50, 20, 9, 77], [128, 128], poison=False)
    for first, shared in (([0, 2**31 - 1, 5], [2**31 - 1] * 5), ([-2**31, 9, -4], [-2**31, 64, 2**30, 0, 100]),
                          ([5, 3, 0], [100] * 5), ([0, 3, 5], [2**31 - 1, 64, 0, -1, 10**6])):
        out, lse = call(torch, a, sharing=g.KVSharing(ints(torch, first), ints(torch, shared)))
        torch.cuda.synchronize()
        assert out.shape == (35, 4, 64) and lse.shape == (35, 4)


def test_tables_with_little_room(torch):
    """The same result, without the groups' own launches; and with a width right at the border."""
    D, KV, page, B = 64, 2, 16, 5
    border = -(-ROOM // (2 * KV * D * page * B))
    for width in (30, border - 1, border):
        a = inputs(torch, 7, "bf16", "bf16", 4, KV, D, page, [3, 2], [1, 1, 2, 1, 30], [40, 50, 20, 9, 77], [256, 160],
                   width=width)
        holds(torch, a, call(torch, a, sharing=sharing(torch, a)))
        assert grouped(a) == (width == border)


def test_rows_past_the_last_start_and_strides(torch):
    a = inputs(torch, 7, "bf16", "bf16", 4, 2, 64, 16, [3, 2], [1, 1, 2, 1, 30], [40, 50, 20, 9, 77], [256, 160])
    want = ref.attend(a)
    n = len(a["q_gpu"])
    wide = torch.full((n + 9, 7, 64), NAN, dtype=torch.bfloat16, device="cuda")
    wide[:n, :4] = a["q_gpu"]
    out = torch.full((n + 9, 9, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    got, lse = call(torch, a, q=wide[:, :4], out=out[:, 2:6], sharing=sharing(torch, a))
    holds(torch, a, (got[:n], lse[:n]), want)
    assert (out[:, :2] == 7).all() and (out[:, 6:] == 7).all() and (out[n:] == 7).all()


def test_same_bits_again_and_in_graphs(torch):
    """Two captured graphs of one cache, other groups for each replay, eager calls between them, another stream."""
    sets = [inputs(torch, 9, "bf16", "mx4", 8, 2, 128, 16, groups, [1, 1, 1, 1, 20], [300, 20, 70, 1, 60], shared, poison=False)
            for groups, shared in (([5], [1024]), ([2, 3], [640, 1024]), ([1, 1, 1, 2], [0, 64, 100, 1008]))]
    cache, q = sets[0]["cache"], sets[0]["q_gpu"]
    most = max(s["tables"].shape[1] for s in sets)

    def given(s):
        t = np.full((5, most), -1)
        t[:, :s["tables"].shape[1]] = s["tables"]
        return ints(torch, s["starts"]), ints(torch, s["lens"]), ints(torch, t)

    held = [list(given(s)) for s in (sets[0], sets[1])]
    step = lambda x, least: cache.attend(q, *x, with_lse=True, sharing=g.kv_share(
        x[2], x[1] - (x[0][1:] - x[0][:-1]), 16, least=least))
    for x in held:
        step(x, 64)
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph, x in zip(graphs, held):
        with torch.cuda.graph(graph):
            outs.append(step(x, 64))
    side = torch.cuda.Stream()
    for s in (sets[1], sets[2], sets[0], sets[1]):
        for x, graph, out in zip(held, graphs, outs):
            for y, z in zip(x, given(s)):
                y.copy_(z)
            for y in out:
                y.fill_(9)
            graph.replay()
            eager = step(x, 64)
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                other = step(x, 64)
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            for y, z, w in zip(out, eager, other):
                assert torch.equal(y, z) and torch.equal(y, w)
        apart = cache.attend(q, *held[0], with_lse=True)
        x, y = out[0].double(), apart[0].double()
        assert (x - y).norm() <= 2 ** -7 * y.norm()


def test_nothing_new_and_refusals(torch):
    a = inputs(torch, 8, "bf16", "bf16", 4, 2, 64, 16, [2], [1, 1], [40, 50], [128], poison=False)
    with pytest.raises(ValueError, match="sharing.shared"):
        call(torch, a, sharing=g.KVSharing(ints(torch, [0, 2]), ints(torch, [128])))
    with pytest.raises(TypeError, match="sharing.first"):
        call(torch, a, sharing=g.KVSharing(ints(torch, [0, 2]).long(), ints(torch, [128, 128])))
    with pytest.raises(g.GorioError, match="groups=0"):
        call(torch, a, sharing=g.KVSharing(ints(torch, [0]), ints(torch, [128, 128])))
    with pytest.raises(g.GorioError, match="groups=3"):
        call(torch, a, sharing=g.KVSharing(ints(torch, [0, 1, 2, 2]), ints(torch, [128, 128])))
    out = a["cache"].attend(a["q_gpu"][:0], ints(torch, [0, 0, 0]), ints(torch, [130, 128]), ints(torch, a["tables"]),
                            sharing=sharing(torch, a))
    assert out.shape == (0, 4, 64)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "mx4"), ("f16", "mx8")])
@pytest.mark.parametrize("D", [64, 96, 128, 192])
def test_shared_values_that_some_rows_see(torch, type, cache, D):
    """NaN and inf among shared values that one request's prefix hides and another's shows."""
    a = inputs(torch, 10, type, cache, 4, 2, D, 16, [3], [1, 2, 20], [30, 40, 50], [320], prefix=[320, 100, 320], poison=False)
    # request 1 sees all up to its own tokens; it and the first end before the shared positions do
    a["lens"] = np.array([350, 160, 370])
    bad, c = 200, a["cache"]
    page, place = a["tables"][0, bad // 16], bad % 16
    hit = np.zeros((23, 4, D), bool)
    sees = np.array([True] + [False] * 2 + [True] * 20)
    if cache in mx.KINDS:
        c.value_scale.view(torch.uint8)[page, 1, place, 1] = 255
        hit[sees, 2:, 32:64] = True
        signs = None
    else:
        c.values[page, 0, place, 3], c.values[page, 1, place, 5] = NAN, float("inf")
        c.values[page, 1, place, D - 1] = float("-inf")
        hit[sees, :2, 3], hit[sees, 2:, 5], hit[sees, 2:, D - 1] = True, True, True
        signs = ((slice(2, 4), 5, np.inf), (slice(2, 4), D - 1, -np.inf))
    assert grouped(a)
    want, _, bound, _ = ref.attend(a)
    out, _ = call(torch, a, sharing=sharing(torch, a))
    x = out.double().cpu().numpy()
    assert (np.abs(x - want)[~hit] <= bound[~hit]).all()
    assert not np.isfinite(x[hit]).any()
    if signs:
        for heads, d, value in signs:
            assert (x[sees][:, heads, d] == value).all()
