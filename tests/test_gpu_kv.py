"""The paged key/value calls on the GPU against plain 64-bit forms."""
import numpy as np
import pytest

import kv_reference as ref
import paper_2607_04415_amd as g

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    torch.cuda.set_device(0)
    return torch


def types(torch):
    return {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}


def ints(torch, a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


# --------------------------------------------------------------------------- #
# attach and plan
# --------------------------------------------------------------------------- #
@pytest.mark.parametrize("B,k,page,width,limit", [
    (1, 1, 16, 8, None), (3, 10, 16, 64, 50), (7, 257, 1, 300, 299), (2, 1024, 5, 2000, 1700), (5, 4, 8, 16, 0),
    (4, 64, 64, 33, 33)])
def test_attach(torch, B, k, page, width, limit):
    rng = np.random.default_rng([B, k, page])
    n = 500
    tokens = rng.integers(0, 4 * page, n).astype(np.int32)
    tokens[rng.integers(0, n, 20)] = 0
    tokens[7] = -5
    first = np.cumsum(rng.integers(1, 9, n)).astype(np.int32)
    nodes = rng.integers(0, n, (B, k)).astype(np.int32)
    nodes[rng.random((B, k)) < 0.1] = -1                # a search's padding, also between ids
    nodes[0, 0] = n                                     # past the directory
    if B > 1:
        nodes[1, 0] = 7
    if B > 2:
        nodes[2] = -1
    got = g.kv_attach(torch.from_numpy(nodes).cuda(), torch.from_numpy(first).cuda(), torch.from_numpy(tokens).cuda(),
                      page, width, limit)
    want = ref.attach(nodes, first, tokens, page, width, width if limit is None else limit)
    for x, y in zip(got, want):
        assert np.array_equal(x.cpu().numpy(), y)


@pytest.mark.parametrize("B,most,page,width,short,extra", [
    (1, 1, 16, 8, 0, 0), (1, 0, 16, 1, 0, 0), (5, 40, 16, 12, 0, 3), (300, 9, 1, 40, 0, 0), (700, 30, 24, 9, 100, 0),
    (3, 5000, 7, 1500, 0, 17), (2, 50, 4, 5, 0, 0), (9, 100, 16, 20, 60, -50), (4, 6, 65536, 2, 0, 0)])
def test_plan(torch, B, most, page, width, short, extra):
    rng = np.random.default_rng([B, most, page])
    before = rng.integers(0, max(1, width * page - most), B).astype(np.int32)
    added = rng.integers(0, most + 1, B).astype(np.int32)
    if B > 3:
        before[1], added[2], before[3], added[3] = 0, 0, -4, -1
        before[0] = width * page - 2                    # its new tokens pass the table's end
    tables = rng.integers(0, 1000, (B, width)).astype(np.int32)
    total = int(np.maximum(added, 0).sum())
    T = max(0, total + extra)
    free = rng.permutation(5 * B + total).astype(np.int32)
    if short:
        free = free[:short]
    want = ref.plan(before, added, free, tables, page, T)
    on = torch.from_numpy(tables.copy()).cuda()
    for _ in range(2):                                  # a second call writes the same
        p = g.kv_plan(torch.from_numpy(before).cuda(), torch.from_numpy(added).cuda(), torch.from_numpy(free).cuda(),
                      on, page, T)
        for x, y in zip((p.starts, p.lens, p.positions, p.slots, on, p.taken), want):
            assert np.array_equal(x.cpu().numpy(), y if isinstance(y, np.ndarray) else [y])


def test_plan_without_free_pages(torch):
    on = torch.full((2, 3), -1, dtype=torch.int32, device="cuda")
    p = g.kv_plan(ints(torch, [0, 3]), ints(torch, [2, 1]), ints(torch, []), on, 4, 3)
    assert p.slots.tolist() == [-1, -1, -1] and p.taken.tolist() == [1] and p.positions.tolist() == [0, 1, 3]


# --------------------------------------------------------------------------- #
# store
# --------------------------------------------------------------------------- #
def e4m3(x):
    """The nearest value of four bits of exponent and three of fraction, ties to even, at most 448."""
    x = np.clip(x, -448, 448)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 1e-30))), -6) - 3)
    return np.round(x / step) * step


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("T,H,D,page,scaled", [(1, 1, 8, 1, False), (37, 2, 64, 16, True), (300, 3, 40, 7, True),
                                               (65, 8, 256, 64, False)])
def test_store(torch, type, cache, T, H, D, page, scaled):
    gen = torch.Generator().manual_seed(T + D)
    t, c = types(torch)[type], types(torch)[cache]
    pages = T // page + 3
    shape = (pages, page, H, D)                         # token-major pages, seen as [page][head][token][D]
    k, v = (torch.full(shape, 3, dtype=torch.uint8 if cache == "e4m3" else c).cuda() for _ in range(2))
    if cache == "e4m3":
        k, v = k.view(c), v.view(c)
    scales = [None, None]
    if cache == "e4m3" and scaled:
        scales = [torch.rand(H, generator=gen).cuda() * 0.02 + 0.004 for _ in range(2)]
    kv = g.KVCache(k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3), *scales)
    rows = (torch.randn(T, 2 * H + 1, D, generator=gen) * 3).to(t)
    rows[0, 1, :4] = torch.tensor([NAN, 70000.0 if type == "bf16" else 60000.0, -60000.0, 0.0], dtype=t)
    rows = rows.cuda()
    slots = torch.randperm(pages * page, generator=gen)[:T]
    slots[T // 2:T // 2 + 1] = -1
    if T > 5:
        slots[2] = pages * page                         # past the last page
        slots[3] = 1 << 40
    before = k.float().cpu().numpy(), v.float().cpu().numpy()
    kv.store(rows[:, 1:1 + H], rows[:, 1 + H:], slots.cuda())
    for pool, had, lo, scale in ((k, before[0], 1, scales[0]), (v, before[1], 1 + H, scales[1])):
        want = had.reshape(-1, H, D).copy()
        x = rows[:, lo:lo + H].float().cpu().numpy()
        if cache == "e4m3":
            # the quotient is rounded to 32 bits first, as stated
            x = e4m3((x / (1 if scale is None else scale.cpu().numpy()[:, None])).astype(np.float32).astype(np.float64))
        for i, s in enumerate(slots.tolist()):
            if 0 <= s < pages * page:
                want[s] = x[i]
        assert np.array_equal(pool.float().cpu().numpy().reshape(-1, H, D), want, equal_nan=True)


@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_store_every_value_in_8_bits(torch, type):
    """All 16-bit values by factors of all sizes: every quotient rounded to 32 bits, then to 8."""
    factors = np.array([1.0, 0.013, 0.7 + 2**-24, 1 - 2**-24, 1 + 2**-23, 3.0, 1 / 448, -0.02, 2.0**-60, 2.0**-61,
                        1.5e-39, 2.0**61, 3e38, 0.0, 7e-7, 1.0625 - 2**-23], np.float32)
    H, D = len(factors), 64
    rows = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(types(torch)[type]).reshape(-1, 1, D)
    T = rows.shape[0]
    k, v = (torch.zeros(T, H, 1, D).to(torch.float8_e4m3fn).cuda() for _ in range(2))
    kv = g.KVCache(k, v, torch.from_numpy(factors).cuda(), torch.from_numpy(factors[::-1].copy()).cuda())
    wide = rows.expand(T, H, D).contiguous().cuda()
    kv.store(wide, wide, torch.arange(T, device="cuda"))
    x = rows.float().numpy()
    with np.errstate(all="ignore"):
        for pool, by in ((k, factors), (v, factors[::-1])):
            want = e4m3((x / by[:, None]).astype(np.float32).astype(np.float64))
            assert np.array_equal(pool.float().cpu().numpy()[:, :, 0], want, equal_nan=True)


# --------------------------------------------------------------------------- #
# attend
# --------------------------------------------------------------------------- #
def setup(torch, seed, type, cache, H, KV, D, page, news, lens, *, fills=False, prefix=None, slopes=False, window=0,
          cap=0.0, scale=None, absent=0.0, token_major=False, poison=True, width=None, spread=1.0):
    """A cache whose pages are spread over the pool, everything that no token may see poisoned with NaN and inf."""
    rng = np.random.default_rng(seed)
    tt = types(torch)
    news, lens = np.array(news), np.array(lens)
    entries = -(-lens // page)
    width = max(1, int(entries.max()) + 1 if len(lens) else 1) if width is None else width
    pages = int(entries.sum()) + 2
    order = rng.permutation(pages)
    tables = np.full((len(lens), width), -1, np.int32)
    at = 0
    for b, e in enumerate(entries):
        e = min(int(e), width)
        tables[b, :e] = order[at:at + e]
        at += e
    gone = rng.random(tables.shape) < absent
    tables[gone] = rng.choice([-1, -2**31, pages, 2**31 - 1], int(gone.sum()))
    a = {"page": page, "D": D, "type": type, "tables": tables, "scale": D ** -0.5 if scale is None else scale,
         "lens": lens, "starts": np.concatenate([[0], np.cumsum(news)]), "window": window, "cap": cap}
    if prefix is not None:
        a["prefix"] = np.array(prefix)
    if fills:
        f = rng.integers(0, page + 1, tables.shape)
        f[rng.random(tables.shape) < 0.4] = page
        a["fills"] = f
    if slopes:
        a["slopes"] = 2.0 ** -np.linspace(1, 8, H)
        a["slopes"][0] = 0.0
    gen = torch.Generator().manual_seed(seed)
    pool, scales = [], []
    for _ in range(2):
        x = torch.randn(pages, KV, page, D, generator=gen) * spread
        s = (torch.rand(KV, generator=gen) * 0.02 + 0.01) if cache == "e4m3" else None
        x = x.to(tt[cache]) if s is None else (x / s[:, None, None]).clamp(-448, 448).to(tt[cache])
        pool.append(x)
        scales.append(s)
    q = (torch.randn(int(news.sum()), H, D, generator=gen) * spread).to(tt[type])
    a["q"] = q.double().numpy()
    for name, x, s in zip(("keys", "values"), pool, scales):
        a[name] = x.double().numpy() * (1.0 if s is None else s.double().numpy()[:, None, None])
    if poison:
        seen = np.zeros((pages, page), bool)
        for b in range(len(lens)):
            n = int(news[b])
            for i in range(n):
                j = ref.visible(b, int(lens[b]) - n + i, int(lens[b]), a)
                seen[tables[b, j // page], j % page] = True
        bad = torch.from_numpy(~seen)[:, None, :, None].expand(pool[0].shape)
        for x in pool:
            f = x.float()
            f[bad] = NAN
            if cache != "e4m3":
                f[:, :, ::2][bad[:, :, ::2]] = float("inf")
            x.copy_(f.to(x.dtype))
    if token_major:                                     # [page][token][head][D] in memory
        pool = [x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) for x in pool]
    else:
        pool = [x.cuda() for x in pool]
    a["cache"] = g.KVCache(*pool, *[None if s is None else s.cuda() for s in scales])
    a["q_gpu"] = q.cuda()
    return a


def call(torch, a, **more):
    given = {k: ints(torch, a[k]) for k in ("fills", "prefix") if a.get(k) is not None}
    if a.get("slopes") is not None:
        given["slopes"] = torch.tensor(a["slopes"], dtype=torch.float32, device="cuda")
    q = more.pop("q", a["q_gpu"])
    return a["cache"].attend(q, ints(torch, a["starts"]), ints(torch, a["lens"]), ints(torch, a["tables"]),
                             scale=a["scale"], cap=a["cap"], window=a["window"], with_lse=True, **given, **more)


def holds(torch, a, got, want=None):
    out, lse = got
    w_out, w_lse, bound, lse_bound = ref.attend(a) if want is None else want
    x, z = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.isfinite(x).all()
    off = np.abs(x - w_out) - bound
    assert (off <= 0).all(), f"off by {np.abs(x - w_out).max()} at {np.unravel_index(off.argmax(), off.shape)}"
    none = np.isneginf(w_lse)
    assert np.array_equal(np.isneginf(z), none)
    assert (np.abs(z - w_lse)[~none] <= lse_bound[~none]).all(), np.abs(z - w_lse)[~none].max()
    assert (x[none] == 0).all()


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("H,KV,D,page", [(1, 1, 8, 1), (4, 4, 64, 16), (8, 2, 128, 16), (6, 1, 96, 3), (3, 3, 40, 7),
                                         (10, 2, 136, 48), (40, 1, 72, 8), (4, 2, 256, 64)])
def test_attend_shapes(torch, type, cache, H, KV, D, page):
    """Single tokens, short chunks, nothing new, lengths of one, and rows with all kinds of ends."""
    a = setup(torch, D + page, type, cache, H, KV, D, page, [1, 5, 0, 1, 33, 2], [1, 5, 9, 130, 97, 64])
    want = ref.attend(a)
    for max_new in (0, 33):
        holds(torch, a, call(torch, a, max_new=max_new), want)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [3, 1, 0, 4], [40, 1, 70, 2]])
@pytest.mark.parametrize("opts", [
    dict(window=1), dict(window=17), dict(cap=20.0), dict(cap=0.5, window=70), dict(slopes=True),
    dict(prefix=[0, 64, 1000, 7]), dict(prefix=[100, 90, 80, 70], window=5), dict(fills=True),
    dict(fills=True, prefix=[96, 0, 64, 200], slopes=True, cap=30.0, window=33), dict(absent=0.5),
    dict(absent=1.0), dict(fills=True, absent=0.3, prefix=[2**31 - 1, -5, 3, 0], slopes=True)])
def test_attend_masks(torch, type, cache, news, opts):
    """Windows, prefixes, caps, biases, pages that end early or are missing, rows that see nothing."""
    a = setup(torch, 3, type, cache, 4, 2, 64, 16, news, [120, 97, 203, 71], **opts)
    holds(torch, a, call(torch, a, max_new=max(news)))


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.5])
@pytest.mark.parametrize("news", [[1, 4], [50, 30]])
def test_attend_scales(torch, news, scale):
    """A factor of 0 (the mean of what is seen), a negative one, one above 1."""
    a = setup(torch, 17, "f16", "f16", 4, 2, 64, 16, news, [150, 130], scale=scale, window=60)
    holds(torch, a, call(torch, a))


@pytest.mark.parametrize("scale,cap", [(0.0, 0.0), (1e-36, 0.0), (-0.3, 0.0), (-0.3, 20.0), (0.0, 5.0), (0.7, 300.0)])
@pytest.mark.parametrize("news", [[1, 4], [50, 30]])
def test_attend_biased_scales(torch, news, scale, cap):
    """Biases beside scores of no size, of both signs, capped and not, before and behind the tokens."""
    a = setup(torch, 23, "f16", "f16", 4, 2, 64, 16, news, [150, 130], scale=scale, cap=cap, slopes=True,
              prefix=[150, 20])
    holds(torch, a, call(torch, a))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("news", [[1, 3], [40, 20]])
def test_attend_biased_from_afar(torch, news, D):
    """All pages near the tokens are missing: the distances are thousands, and so are the biases."""
    a = setup(torch, D + 1, "f16", "f16", 2, 1, D, 16, news, [6000, 3001], slopes=True, poison=False)
    a["tables"][:, 6:] = -1
    a["slopes"] = [0.0, 0.5]
    holds(torch, a, call(torch, a))


@pytest.mark.parametrize("news", [[1, 1], [50, 3]])
def test_attend_table_narrower_than_the_length(torch, news):
    a = setup(torch, 5, "bf16", "bf16", 4, 2, 64, 16, news, [150, 130], width=3)
    holds(torch, a, call(torch, a))


@pytest.mark.parametrize("news", [[1, 2], [90, 11]])
def test_attend_strides(torch, news):
    """Token-major pages, queries and outputs that are parts of wider rows."""
    a = setup(torch, 6, "bf16", "bf16", 8, 2, 64, 16, news, [150, 130], token_major=True)
    T = len(a["q"])
    wide = torch.full((T, 12, 64), NAN, dtype=torch.bfloat16, device="cuda")
    wide[:, :8] = a["q_gpu"]
    out = torch.full((T, 11, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    got = call(torch, a, q=wide[:, :8], out=out[:, 2:10])
    holds(torch, a, got)
    assert (out[:, :2] == 7).all() and (out[:, 10:] == 7).all()


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("news,lens,H,KV", [([1], [9000], 2, 1), ([2, 1, 1], [5000, 3, 2500], 4, 2),
                                            ([20, 1], [4100, 700], 2, 2)])
def test_attend_long(torch, type, cache, news, lens, H, KV):
    """Few rows over long texts: the keys are divided and the parts joined."""
    a = setup(torch, 8, type, cache, H, KV, 64, 16, news, lens, fills=True, prefix=[n // 2 for n in lens])
    holds(torch, a, call(torch, a, max_new=max(news)))


@pytest.mark.parametrize("B,most,longest", [(1300, 1, 60), (700, 1, 900), (600, 3, 100), (300, 90, 130)])
def test_attend_many_requests(torch, B, most, longest):
    """More requests, and more tiles, than a workgroup has threads; some with nothing new or nothing at all."""
    rng = np.random.default_rng([B, most])
    news = rng.integers(0, most + 1, B) if most > 1 else np.ones(B, int)
    if most > 50:
        news[rng.random(B) < 0.9] = 1
    lens = np.maximum(news, rng.integers(0, longest, B))
    lens[5] = longest + 700
    a = setup(torch, B, "bf16", "bf16", 2, 1, 64, 16, news, lens, poison=False)
    holds(torch, a, call(torch, a, max_new=int(news.max())))


def test_attend_more_key_heads_than_workgroups(torch):
    a = setup(torch, 18, "f16", "f16", 300, 300, 8, 16, [1, 70], [600, 90], poison=False)
    holds(torch, a, call(torch, a))


@pytest.mark.parametrize("D", [64, 96, 128, 200])
def test_attend_cut_tiles(torch, D):
    """Chunks over texts long enough that their tiles are divided among workgroups."""
    a = setup(torch, D, "bf16", "bf16", 2, 1, D, 16, [9, 40], [2600, 1500], fills=True, slopes=True)
    holds(torch, a, call(torch, a))


@pytest.mark.parametrize("news", [[1, 3], [64, 40]])
def test_attend_peaked(torch, news):
    """Scores of several hundred, of both signs: the running maximum moves by a lot."""
    a = setup(torch, 9, "f16", "f16", 4, 2, 64, 16, news, [300, 260], spread=7.0)
    holds(torch, a, call(torch, a))


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("news", [[3], [100]])
def test_attend_future_values_do_not_reach_a_row(torch, type, news):
    """A later token of the same chunk holds NaN and inf: earlier rows do not see it, and later ones do."""
    n = news[0]
    a = setup(torch, 10, type, type, 4, 2, 64, 16, news, [150], poison=False)
    bad = 150 - n // 2                                  # visible to the last n // 2 rows only
    page, place = a["tables"][0, bad // 16], bad % 16
    a["cache"].values[page, 0, place, 3] = NAN
    a["cache"].values[page, 1, place, 5] = float("inf")
    a["cache"].values[page, 1, place, 9] = float("-inf")
    out, _ = call(torch, a)
    w_out, _, bound, _ = ref.attend(a)
    x = out.double().cpu().numpy()
    sees = np.arange(n) >= n - n // 2
    hit = np.zeros((n, 4, 64), bool)
    hit[sees, :2, 3], hit[sees, 2:, 5], hit[sees, 2:, 9] = True, True, True
    assert np.isnan(x[sees][:, :2, 3]).all()
    assert np.isposinf(x[sees][:, 2:, 5]).all() and np.isneginf(x[sees][:, 2:, 9]).all()
    assert (np.abs(x - w_out)[~hit] <= bound[~hit]).all()


def test_attend_nan_and_inf_scores(torch):
    """What a row does see reaches it: a NaN key, a score of inf; keys at -inf weigh nothing."""
    a = setup(torch, 11, "bf16", "bf16", 2, 1, 64, 16, [1, 1, 1, 40], [70, 70, 70, 90], poison=False)
    keys = a["cache"].keys
    at = lambda b, j: (a["tables"][b, j // 16], 0, j % 16)
    keys[at(0, 5)] = NAN
    keys[at(1, 5)] = a["q_gpu"][1, 0].sign() * float("inf")          # head 0: +inf, head 1: NaN or inf
    keys[at(2, 5)] = -a["q_gpu"][2, 0].sign() * float("inf")         # head 0: -inf
    out, lse = call(torch, a)
    x = out.float().cpu().numpy()
    assert np.isnan(x[0]).all() and np.isnan(lse[0].cpu().numpy()).all()
    assert np.isnan(x[1, 0]).all()
    a["keys"][at(2, 5)] = -1e30 * np.sign(a["q"][2, 0])
    w_out, _, bound, _ = ref.attend(a)
    assert (np.abs(x[2, 0] - w_out[2, 0]) <= bound[2, 0]).all()
    assert (np.abs(x[3:] - w_out[3:]) <= bound[3:]).all()


def test_attend_all_scores_minus_inf(torch):
    a = setup(torch, 12, "bf16", "bf16", 1, 1, 64, 16, [1], [1], poison=False)
    a["cache"].keys[:] = (-a["q_gpu"][0, 0].sign() * float("inf"))[None, None, None]
    out, lse = call(torch, a)
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_attend_past_32_bits(torch):
    """Pages whose offsets pass 2^32 bytes and 2^32 elements."""
    pages, page, D = 140_000, 256, 128                  # 9.2 GB for the keys
    k = torch.empty((pages, 1, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    table = np.array([[pages - 1, 3, pages - 2, 70_000]])
    gen = torch.Generator(device="cuda").manual_seed(1)
    for x in (k, v):
        for p in table[0]:
            x[p] = torch.randn((1, page, D), generator=gen, device="cuda").bfloat16()
    small = [torch.stack([x[p] for p in table[0]]).double().cpu().numpy() for x in (k, v)]
    cache = g.KVCache(k, v)
    rows = torch.randn((2, 1, D), generator=gen, device="cuda").bfloat16()
    slots = torch.tensor([(pages - 2) * page + 255, 70_000 * page + 9], device="cuda")
    cache.store(rows, rows * 2, slots)
    small[0][2, 0, 255], small[0][3, 0, 9] = rows[:, 0].double().cpu().numpy()
    small[1][2, 0, 255], small[1][3, 0, 9] = (rows * 2)[:, 0].double().cpu().numpy()
    for n in (1, 40):
        q = torch.randn((n, 2, D), generator=gen, device="cuda").bfloat16()
        a = {"page": page, "D": D, "type": "bf16", "tables": np.arange(4)[None], "scale": D ** -0.5, "cap": 0.0,
             "lens": np.array([900]), "starts": np.array([0, n]), "window": 0, "q": q.double().cpu().numpy(),
             "keys": small[0], "values": small[1]}
        got = cache.attend(q, ints(torch, [0, n]), ints(torch, [900]), ints(torch, table), with_lse=True)
        holds(torch, a, got)


def test_attend_rows_past_the_last_start(torch):
    """starts that end before the rows do, or past them: no row but the named ones is written."""
    a = setup(torch, 13, "bf16", "bf16", 2, 1, 64, 16, [3, 4], [50, 60])
    want = ref.attend(a)
    q = torch.cat([a["q_gpu"], a["q_gpu"]])
    out = torch.full_like(q, 5.0)
    got, lse = call(torch, a, q=q, out=out)
    holds(torch, a, (got[:7], lse[:7]), want)
    assert (got[7:] == 5).all()


def test_attend_same_bits_again_on_another_stream_and_in_a_graph(torch):
    a = setup(torch, 14, "bf16", "bf16", 8, 2, 128, 16, [1, 1, 1, 30], [3000, 700, 1, 900], poison=False)
    first = [x.clone() for x in call(torch, a)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = call(torch, a)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(first, again))
    # a step as a program captures it: plan, store, attend
    rng = np.random.default_rng(14)
    news, before = [1, 2, 20], [100, 33, 5]
    cache = a["cache"]
    free = torch.arange(150, 200, dtype=torch.int32, device="cuda")
    tables = torch.zeros((3, 12), dtype=torch.int32, device="cuda")
    tables[:] = torch.arange(36, device="cuda").view(3, 12)
    k = torch.randn(23, 2, 128, device="cuda").bfloat16()
    q = torch.randn(23, 8, 128, device="cuda").bfloat16()
    b, n = ints(torch, before), ints(torch, news)

    def step():
        p = g.kv_plan(b, n, free, tables, 16, 23)
        cache.store(k, k, p.slots)
        return cache.attend(q, p.starts, p.lens, tables, max_new=20)

    eager = step().clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        k.copy_(torch.randn(23, 2, 128, device="cuda").bfloat16())
        out.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step()), i
    assert not torch.equal(eager, got)


def test_attend_nothing(torch):
    a = setup(torch, 15, "bf16", "bf16", 2, 1, 64, 16, [0, 0], [5, 0])
    out, lse = call(torch, a)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)


# --------------------------------------------------------------------------- #
# refusals
# --------------------------------------------------------------------------- #
def test_refusals(torch):
    a = setup(torch, 16, "bf16", "bf16", 4, 2, 64, 16, [2], [20])
    cache, q = a["cache"], a["q_gpu"]
    starts, lens, tables = ints(torch, [0, 2]), ints(torch, [20]), ints(torch, a["tables"])
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        cache.attend(q.float(), starts, lens, tables)
    with pytest.raises(g.GorioError, match="own type"):
        cache.attend(q.half(), starts, lens, tables)
    with pytest.raises(g.GorioError, match="multiple of the cache's"):
        cache.attend(q[:, :3].contiguous(), starts, lens, tables)
    with pytest.raises(ValueError, match="starts"):
        cache.attend(q, lens, lens, tables)
    with pytest.raises(ValueError, match="on cuda"):
        cache.attend(q, starts.cpu(), lens, tables)
    with pytest.raises(g.GorioError, match="cap"):
        cache.attend(q, starts, lens, tables, cap=-1.0)
    with pytest.raises(g.GorioError, match="cap"):
        cache.attend(q, starts, lens, tables, cap=NAN)
    with pytest.raises(ValueError, match="contiguous"):
        cache.attend(q[:, ::2], starts, lens, tables)
    odd = torch.zeros(2 * 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 4, 64)
    with pytest.raises(g.GorioError, match="multiple of 16 bytes"):
        cache.attend(odd, starts, lens, tables)
    with pytest.raises(TypeError, match="slots"):
        cache.store(q[:, :2], q[:, :2], starts)
    with pytest.raises(g.GorioError, match="own type"):
        cache.store(q[:, :2].half(), q[:, :2].half(), starts[:2].long())
    with pytest.raises(ValueError, match="float8"):
        g.KVCache(cache.keys, cache.values, key_scale=torch.ones(2, device="cuda"))
    with pytest.raises(TypeError):
        g.KVCache(cache.keys.float(), cache.values.float())
    with pytest.raises(g.GorioError, match="limit"):
        g.kv_attach(ints(torch, [[0]]), lens, lens, 16, 4, 5)
    with pytest.raises(g.GorioError, match="page_tokens"):
        g.kv_plan(lens, lens, lens, tables, 0, 3)
    host = np.zeros(4, np.int32).ctypes.data
    assert g.lib().gorio_kv_plan(host, lens.data_ptr(), 1, 16, None, 0, tables.data_ptr(), 1, 0, starts.data_ptr(),
                                 starts.data_ptr(), None, None, None, None) == g.EINVAL
    assert b"device pointer" in g.lib().gorio_last_error()


def test_attach_without_passages(torch):
    none = ints(torch, [])
    tables, fills, lens, attached = g.kv_attach(ints(torch, [[-1, 3], [0, -1]]), none, none, 16, 4)
    assert (tables == -1).all() and (fills == 16).all() and not lens.any() and not attached.any()


@pytest.mark.parametrize("H,KV", [(2, 2), (8, 2), (17, 1)])
@pytest.mark.parametrize("news,rows,max_new", [
    ([1], 8, 1), ([1, 1, 0, 1], 64, 1), ([2, 1], 30, 2), ([1, 4], 40, 4),       # rows past the last start
    ([1, 40], 41, 1), ([30], 30, 2), ([3, 1, 25], 60, 3)])                      # a hint that is too small
def test_attend_rows_beyond_the_hint(torch, H, KV, news, rows, max_new):
    """A batch padded to a fixed number of rows, and hints that are wrong: the named rows are all computed."""
    a = setup(torch, 19, "bf16", "bf16", H, KV, 64, 16, news, [700, 90, 33, 640][:len(news)])
    n = len(a["q"])
    q = torch.zeros((rows, H, 64), dtype=torch.bfloat16, device="cuda")
    q[:n] = a["q_gpu"]
    out = torch.full_like(q, 5.0)
    got, lse = call(torch, a, q=q, out=out, max_new=max_new)
    holds(torch, a, (got[:n], lse[:n]))
    assert (got[n:] == 5).all()


@pytest.mark.parametrize("B,k", [(1, 4), (3, 300)])
def test_attach_passes_over_passages_without_pages(torch, B, k):
    """A first page below 0: as if the id were not there.  Pages past the largest name none."""
    rng = np.random.default_rng([B, k])
    n, page, width = 60, 8, 700
    tokens = rng.integers(0, 4 * page, n).astype(np.int32)
    first = rng.integers(0, 1000, n).astype(np.int32)
    first[::3] = -1
    first[4] = -2**31
    nodes = rng.integers(0, n, (B, k)).astype(np.int32)
    nodes[:, :4] = [3, 4, 5, 6]
    want = ref.attach(np.where(first[nodes] < 0, -1, nodes), first, tokens, page, width, width)
    got = g.kv_attach(ints(torch, nodes), ints(torch, first), ints(torch, tokens), page, width)
    for x, y in zip(got, want):
        assert np.array_equal(x.cpu().numpy(), y)
    tables, fills, lens, _ = g.kv_attach(ints(torch, [[0]]), ints(torch, [2**31 - 2]), ints(torch, [4 * page]), page, 6)
    assert tables.tolist() == [[2**31 - 2, 2**31 - 1, -1, -1, -1, -1]] and lens.tolist() == [4 * page]


def test_arrays_that_are_written_overlap_no_other(torch):
    """Blocks run in any order: lens where added lies would be read by one after another has written it."""
    L, B, width, T = g.lib(), 3, 4, 6
    x = ints(torch, np.zeros(200))
    at = lambda i: x.data_ptr() + 4 * i
    plan = dict(before=at(0), added=at(3), free=at(8), tables=at(20), lens=at(40), starts=at(44), positions=at(50),
                slots=at(60), taken=at(80))

    def status(**more):
        a = {**plan, **more}
        return L.gorio_kv_plan(a["before"], a["added"], B, 16, a["free"], 5, a["tables"], width, T, a["lens"],
                               a["starts"], a["positions"], a["slots"], a["taken"], None)

    assert status() == g.OK and status(positions=None, slots=None, taken=None) == g.OK
    assert L.gorio_kv_plan(at(0), at(3), B, 16, at(21), 0, at(20), width, T, at(40), at(44), at(50), at(60), at(80),
                           None) == g.OK              # no free page, wherever it points
    for name, where in (("lens", at(3)), ("lens", at(5)), ("starts", at(2)), ("starts", at(42)), ("tables", at(12)),
                        ("positions", at(19)), ("slots", at(52)), ("taken", at(31)), ("taken", at(4))):
        assert status(**{name: where}) == g.EINVAL, (name, where)
        assert b"overlap" in L.gorio_last_error()
    attach = lambda tables, fills, lens, attached: L.gorio_kv_attach(
        at(0), B, 2, at(10), at(20), 5, 16, width, width, tables, fills, lens, attached, None)
    assert attach(at(30), at(42), at(54), at(57)) == g.OK and attach(at(30), at(42), at(54), None) == g.OK
    for arrays in ((at(5), at(42), at(54), at(57)), (at(30), at(41), at(54), at(57)), (at(30), at(42), at(24), at(57)),
                   (at(30), at(42), at(54), at(56))):
        assert attach(*arrays) == g.EINVAL and b"overlap" in L.gorio_last_error()
    torch.cuda.synchronize()
    empty = [torch.empty(0, dtype=torch.int32, device="cuda") for _ in range(2)]
    p = g.kv_plan(ints(torch, [0]), ints(torch, [0]), empty[0], ints(torch, [[-1]]), 16, 0)
    assert p.lens.tolist() == [0] and p.taken.tolist() == [0]
