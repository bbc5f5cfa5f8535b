"""Pages of 8 and 4 bits whose elements share a power of two by blocks of 32: stores, loads, attention.

Stores and loads are exact; attention is held to the bounds of kv_reference.attend, over the
values that the elements stand for, as the queries' type has them."""
import numpy as np
import pytest

import kv_reference as ref
import mx_reference as mx
import paper_2607_04415_amd as g
from test_gpu_kv import call, holds, ints, setup, types

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def pool(torch, kind, code, powers):
    """The tensors of one side of a cache."""
    type = torch.float8_e4m3fn if kind == "mx8" else torch.float4_e2m1fn_x2
    return (torch.from_numpy(code).cuda().view(type), torch.from_numpy(powers).cuda().view(torch.float8_e8m0fnu))


def empty(torch, kind, pages, heads, page, D, fill=0):
    """A cache, and its bytes: keys, key powers, values, value powers."""
    sides = [pool(torch, kind, np.full((pages, heads, page, D // 2 if kind == "mx4" else D), fill, np.uint8),
                  np.full((pages, heads, page, D // 32), fill, np.uint8)) for _ in range(2)]
    (k, kp), (v, vp) = sides
    return g.KVCache(k, v, kp, vp), [x.view(torch.uint8) for x in (k, kp, v, vp)]


def rows(torch, x, type):
    return torch.from_numpy(np.asarray(x, np.float64)).to(types(torch)[type])


# --------------------------------------------------------------------------- #
# store
# --------------------------------------------------------------------------- #
@pytest.mark.parametrize("kind", ["mx8", "mx4"])
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("H,D,page,T", [(1, 32, 1, 1), (2, 64, 16, 37), (3, 96, 24, 50), (8, 128, 16, 5), (1, 160, 7, 333),
                                        (5, 256, 64, 70)])
def test_store(torch, kind, type, H, D, page, T):
    """Rows of a fused projection with sizes from 2^-30 to 2^15, zeros among them, into scattered slots; some
    name no page, and no other byte changes."""
    rng = np.random.default_rng([H, D, T])
    pages = -(-T // page) + 2
    cache, had = empty(torch, kind, pages, H, page, D, fill=77)
    x = rng.standard_normal((T, 1 + 2 * H, D)) * 2.0 ** rng.uniform(-30, 12, (T, 1 + 2 * H, 1))
    x[rng.random(x.shape) < 0.1] = 0
    x[0, :, :32] = 0
    x = rows(torch, x, type)
    slots = rng.permutation(pages * page)[:T]
    out = rng.random(T) < 0.2
    slots[out] = rng.choice([-1, -2**40, pages * page, 2**40, 2**31 + 5], int(out.sum()))
    cache.store(x[:, 1:1 + H].cuda(), x[:, 1 + H:].cuda(), torch.from_numpy(slots).cuda())
    for i, lo in ((0, 1), (2, 1 + H)):
        code, powers = mx.pack(x[:, lo:lo + H].double().numpy(), kind)
        for got, want in ((had[i], code), (had[i + 1], powers)):
            got = got.cpu().numpy().swapaxes(1, 2).reshape(pages * page, H, -1)
            all = np.full_like(got, 77)
            for t in range(T):
                if 0 <= slots[t] < pages * page:
                    all[slots[t]] = want[t]
            assert np.array_equal(got, all)


@pytest.mark.parametrize("kind", ["mx8", "mx4"])
@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_store_every_value(torch, kind, type):
    """Every 16-bit value, subnormal, infinite and NaN ones too, as its block's largest and beside a larger one."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(types(torch)[type])
    x = torch.zeros(65536, 4, 32, dtype=bits.dtype)
    x[:, 0, 5] = bits                                                   # the largest of its block
    x[:, 0, 20] = bits * 0.3
    x[:, 1] = bits[:, None]
    x[:, 2, 0], x[:, 2, 31] = bits, bits * 5
    x[:, 3, 7], x[:, 3, 8] = bits, 1.0
    cache, had = empty(torch, kind, 65536, 4, 1, 32)
    cache.store(x.cuda(), x.cuda(), torch.arange(65536, device="cuda"))
    wide = x.double().numpy()
    finite = np.isfinite(wide).all(-1)
    p = mx.powers_of(wide, kind).astype(int)
    u = np.where(finite[..., None], wide, 0) / 2.0 ** (p - 127.0)[..., None]
    code = mx.nearest(u, kind)
    code[~finite] = 0
    code = code[..., ::2] | code[..., 1::2] << 4 if kind == "mx4" else code
    for got, want in zip(had, (code, p[..., None], code, p[..., None])):
        assert np.array_equal(got.cpu().numpy()[:, :, 0], want)


# --------------------------------------------------------------------------- #
# load
# --------------------------------------------------------------------------- #
@pytest.mark.parametrize("kind", ["mx8", "mx4"])
@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_load_every_element(torch, kind, type):
    """All codes under all powers, to the nearest 16-bit value."""
    codes = np.arange(256, dtype=np.uint8)
    D = 256
    code = np.tile(codes[:D // 2] if kind == "mx4" else codes, (512, 1, 1, 1)).reshape(512, 1, 1, -1).copy()
    if kind == "mx4":
        code[256:] = codes[128:]
    powers = np.repeat(np.arange(512) % 256, D // 32).reshape(512, 1, 1, -1).astype(np.uint8)
    assert len(np.unique(code)) == 256
    (k, kp), (v, vp) = pool(torch, kind, code, powers), pool(torch, kind, code[::-1].copy(), powers[::-1].copy())
    cache = g.KVCache(k, v, kp, vp)
    keys, values = cache.load(torch.arange(512, device="cuda"), types(torch)[type])
    for got, c, p in ((keys, code, powers), (values, code[::-1], powers[::-1])):
        want = mx.unpack(c[:, :, 0], p[:, :, 0], kind)
        want = torch.from_numpy(want).to(types(torch)[type])
        assert got.dtype == want.dtype and torch.equal(got.cpu().isnan(), want.isnan())
        assert torch.equal(got.cpu().nan_to_num(0.5), want.nan_to_num(0.5))


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3"),
                                        ("bf16", "mx8"), ("f16", "mx4")])
@pytest.mark.parametrize("H,D,page,T", [(1, 32, 1, 1), (2, 64, 16, 37), (3, 96, 24, 1000), (5, 160, 7, 12)])
def test_load(torch, type, cache, H, D, page, T):
    """Slots in any order, one several times, some outside; into rows of their own and parts of wider ones."""
    rng = np.random.default_rng([H, D, T])
    pages, t = 9, types(torch)[type]
    x = rng.standard_normal((2, pages, H, page, D))
    if cache in mx.KINDS:
        packed = [mx.pack(y, cache) for y in x]
        (k, kp), (v, vp) = (pool(torch, cache, *y) for y in packed)
        kv = g.KVCache(k, v, kp, vp)
        want = [mx.unpack(*y, cache) for y in packed]
    else:
        k, v = (torch.from_numpy(y).float().to(types(torch)[cache]) for y in x)
        scale = torch.rand(H) + 0.5 if cache == "e4m3" else None
        kv = g.KVCache(k.cuda(), v.cuda(), None if scale is None else scale.cuda(), None)
        # one product in 32 bits
        want = [k.float() if scale is None else k.float() * scale[:, None, None], v.float()]
        want = [y.double().numpy() for y in want]
    slots = rng.integers(0, pages * page, T)
    out = rng.random(T) < 0.2
    slots[out] = rng.choice([-1, -2**40, pages * page, 2**40, 2**31 + 5], int(out.sum()))
    s = torch.from_numpy(slots).cuda()
    wide = torch.full((T, 2 * H + 1, D), 7.0, dtype=t, device="cuda")
    for got in (kv.load(s, t), kv.load(s, keys=wide[:, :H], values=wide[:, H + 1:])):
        for y, w in zip(got, want):
            w = w.swapaxes(1, 2).reshape(pages * page, H, D)[np.clip(slots, 0, pages * page - 1)]
            w[(slots < 0) | (slots >= pages * page)] = 0
            assert torch.equal(y.cpu(), torch.from_numpy(w).float().to(t))
    assert (wide[:, H] == 7).all()


def test_load_what_was_stored(torch):
    """A copy of passages from one cache to another, of another kind; token-major pages."""
    gen = torch.Generator().manual_seed(5)
    H, D, page, pages, T = 4, 128, 16, 30, 300
    x = torch.randn(T, 2 * H, D, generator=gen).bfloat16().cuda()
    sides = []
    for _ in range(2):
        e = torch.zeros(pages, page, H, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        p = torch.zeros(pages, page, H, D // 32, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
        sides.append((e.permute(0, 2, 1, 3), p.permute(0, 2, 1, 3)))
    first = g.KVCache(sides[0][0], sides[1][0], sides[0][1], sides[1][1])
    second, _ = empty(torch, "mx8", pages, H, page, D)
    slots = torch.randperm(pages * page, generator=gen)[:T].cuda()
    other = torch.randperm(pages * page, generator=gen)[:T].cuda()
    first.store(x[:, :H], x[:, H:], slots)
    k, v = first.load(slots)
    second.store(k, v, other)
    assert all(torch.equal(a, b) for a, b in zip((k, v), second.load(other)))    # what is exact stays so
    for got, lo in ((k, 0), (v, H)):
        y = x[:, lo:lo + H].double()
        off = (got.double() - y).abs().reshape(T, H, -1, 32)
        # steps of 2^-3 of an element's power of two, or of the block's smallest: half of one
        a = y.abs().reshape(T, H, -1, 32)
        assert (off <= torch.maximum(a * 2.0 ** -4, a.amax(-1, keepdim=True) / 224 * 2.0 ** -10)).all()


def test_store_and_load_past_32_bits(torch):
    """Pages whose offsets pass 2^32 elements, in bytes and in halves of them."""
    pages, page, D = 160_000, 256, 128
    for kind in ("mx4", "mx8"):
        shape = (pages, 1, page, D // 2 if kind == "mx4" else D)
        type = torch.float4_e2m1fn_x2 if kind == "mx4" else torch.float8_e4m3fn
        e = [torch.empty(shape, dtype=torch.uint8, device="cuda") for _ in range(2)]
        p = [torch.empty((pages, 1, page, D // 32), dtype=torch.uint8, device="cuda") for _ in range(2)]
        cache = g.KVCache(e[0].view(type), e[1].view(type), *[y.view(torch.float8_e8m0fnu) for y in p])
        x = torch.randn(4, 1, D, generator=torch.Generator().manual_seed(3)).bfloat16()
        slots = torch.tensor([pages * page - 1, 5, (pages - 2) * page + 7, 140_000 * page], device="cuda")
        cache.store(x.cuda(), (2 * x).cuda(), slots)
        for got, y in zip(cache.load(slots), (x, 2 * x)):
            want = mx.unpack(*mx.pack(y.double().numpy(), kind), kind)
            assert np.array_equal(got.double().cpu().numpy(), want)
        for n in (1, 40):                       # a table of the pages that hold them
            fills = np.zeros((1, 4), int)
            fills[0] = [256, 6, 8, 1]
            table = np.array([[pages - 1, 0, pages - 2, 140_000]])
            for y in (*e, *p):
                for at in table[0]:
                    y[at] = torch.randint(90, 130, y[at].shape, device="cuda").byte() if y.shape[-1] == D // 32 else \
                        torch.randint(0, 120, y[at].shape, device="cuda").byte()
            small = [mx.unpack(y[table[0]].cpu().numpy(), z[table[0]].cpu().numpy(), kind) for y, z in zip(e, p)]
            q = torch.randn((n, 2, D), device="cuda").bfloat16()
            a = {"page": page, "D": D, "type": "bf16", "tables": np.arange(4)[None], "scale": 0.0002, "cap": 0.0,
                 "lens": np.array([900]), "starts": np.array([0, n]), "window": 0, "q": q.double().cpu().numpy(),
                 "keys": small[0], "values": small[1], "fills": fills}
            got = cache.attend(q, ints(torch, [0, n]), ints(torch, [900]), ints(torch, table), fills=ints(torch, fills),
                               scale=0.0002, with_lse=True)
            holds(torch, a, got)
        del cache, e, p
        torch.cuda.empty_cache()


# --------------------------------------------------------------------------- #
# attend
# --------------------------------------------------------------------------- #
def small(torch, kind, seed, type, H, KV, D, *rest, **more):
    """test_gpu_kv's inputs, with its pages (poison and all) packed."""
    a = setup(torch, seed, type, type, H, KV, D, *rest, **more)
    old = a["cache"]
    sides = []
    for name, x in (("keys", old.keys), ("values", old.values)):
        code, powers = mx.pack(x.double().cpu().numpy(), kind)
        y = mx.unpack(code, powers, kind)
        a[name] = torch.from_numpy(np.nan_to_num(y)).to(types(torch)[type]).double().numpy()
        if x.stride(1) != x.shape[2] * x.stride(2):                    # token-major
            code, powers = (np.ascontiguousarray(z.swapaxes(1, 2)) for z in (code, powers))
            sides.append([z.permute(0, 2, 1, 3) for z in pool(torch, kind, code, powers)])
        else:
            sides.append(pool(torch, kind, code, powers))
    a["cache"] = g.KVCache(sides[0][0], sides[1][0], sides[0][1], sides[1][1])
    return a


@pytest.mark.parametrize("kind", ["mx8", "mx4"])
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("H,KV,D,page", [(1, 1, 32, 1), (4, 4, 64, 16), (8, 2, 128, 16), (6, 1, 96, 3), (10, 2, 160, 48),
                                         (20, 1, 224, 8), (4, 2, 256, 64)])
def test_attend_shapes(torch, kind, type, H, KV, D, page):
    """Single tokens, short chunks, nothing new, lengths of one, and rows with all kinds of ends."""
    a = small(torch, kind, D + page, type, H, KV, D, page, [1, 5, 0, 1, 33, 2], [1, 5, 9, 130, 97, 64])
    want = ref.attend(a)
    for max_new in (0, 33):
        holds(torch, a, call(torch, a, max_new=max_new), want)


@pytest.mark.parametrize("kind,type", [("mx4", "bf16"), ("mx8", "f16")])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [3, 1, 0, 4], [40, 1, 70, 2]])
@pytest.mark.parametrize("opts", [
    dict(window=17), dict(cap=20.0), dict(cap=0.5, window=70), dict(cap=300.0), dict(slopes=True),
    dict(prefix=[100, 90, 80, 70], window=5), dict(fills=True, prefix=[96, 0, 64, 200], slopes=True, cap=30.0, window=33),
    dict(absent=0.5), dict(absent=1.0), dict(fills=True, absent=0.3, prefix=[2**31 - 1, -5, 3, 0], slopes=True),
    dict(slopes=True, cap=100.0), dict(scale=-0.3, slopes=True), dict(scale=0.0), dict(scale=0.0, slopes=True)])
@pytest.mark.parametrize("D", [64, 160])
def test_attend_masks(torch, kind, type, news, opts, D):
    """Windows, prefixes, caps, biases, factors, pages that end early or are missing, rows that see nothing."""
    a = small(torch, kind, 3, type, 4, 2, D, 16, news, [120, 97, 203, 71], **opts)
    holds(torch, a, call(torch, a, max_new=max(news)))


@pytest.mark.parametrize("kind", ["mx8", "mx4"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("news,lens,H,KV", [([1], [5000], 2, 1), ([2, 1, 1], [2600, 3, 1300], 4, 2), ([20, 1], [2100, 700], 2, 2),
                                            ([9, 40], [2600, 1500], 2, 1)])
def test_attend_long(torch, kind, D, news, lens, H, KV):
    """The keys are divided and the parts joined."""
    a = small(torch, kind, 8, "bf16", H, KV, D, 16, news, lens, fills=True, prefix=[n // 2 for n in lens], poison=False)
    holds(torch, a, call(torch, a, max_new=max(news)))


@pytest.mark.parametrize("kind", ["mx8", "mx4"])
@pytest.mark.parametrize("news", [[1, 2], [90, 11]])
def test_attend_token_major(torch, kind, news):
    a = small(torch, kind, 6, "bf16", 8, 2, 96, 16, news, [150, 130], token_major=True)
    holds(torch, a, call(torch, a))


@pytest.mark.parametrize("kind", ["mx8", "mx4"])
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("news", [[3], [100]])
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
def test_attend_nan_blocks(torch, kind, type, news, D):
    """A block of a later token's values is NaN: rows that do not see it are as without, those that do
    are NaN at its elements.  And a block of keys: those that see it are NaN throughout."""
    n = news[0]
    for side in (3, 1):
        a = small(torch, kind, 10, type, 4, 2, D, 16, news, [150], poison=False)
        cache = a["cache"]
        bad = 150 - n // 2                                  # visible to the last n // 2 rows only
        page, place = a["tables"][0, bad // 16], bad % 16
        (cache.value_scale if side == 3 else cache.key_scale).view(torch.uint8)[page, 1, place, 1] = 255
        out, _ = call(torch, a)
        w_out, _, bound, _ = ref.attend(a)
        x = out.double().cpu().numpy()
        sees = np.arange(n) >= n - n // 2
        hit = np.zeros((n, 4, D), bool)
        hit[sees, 2:, 32 if side == 3 else 0:64 if side == 3 else D] = True
        assert np.isnan(x[hit]).all()
        assert (np.abs(x - w_out)[~hit] <= bound[~hit]).all()


def test_attend_smallest_and_largest_powers(torch):
    """Powers of 2^-127 and of 2^100 beside each other in bf16: no element is lost or clamped."""
    a = small(torch, "mx8", 12, "bf16", 2, 1, 64, 16, [1, 20], [70, 90], poison=False)
    cache = a["cache"]
    for scale, name in ((cache.key_scale, "keys"), (cache.value_scale, "values")):
        b = scale.view(torch.uint8)
        b[..., 0] = 0
        b[:, :, ::3, 1] = 117 if name == "keys" else 127 + 100
        code = getattr(cache, name).view(torch.uint8).cpu().numpy()
        a[name] = mx.unpack(code, b.cpu().numpy(), "mx8")
    holds(torch, a, call(torch, a))


def test_a_step_in_a_graph_and_on_another_stream(torch):
    """Store, attend and load captured together, replayed with other rows."""
    H, KV, D = 8, 2, 128
    cache, _ = empty(torch, "mx4", 40, KV, 16, D)
    news, before = [1, 2, 20], [100, 33, 5]
    free = torch.arange(30, 40, dtype=torch.int32, device="cuda")
    tables = torch.arange(30, device="cuda").int().view(3, 10).contiguous()
    fill = torch.randn(30 * 16, 2 * KV, D, device="cuda").bfloat16()
    cache.store(fill[:, :KV], fill[:, KV:], torch.arange(30 * 16, device="cuda"))
    k, q = torch.randn(23, KV, D, device="cuda").bfloat16(), torch.randn(23, H, D, device="cuda").bfloat16()
    b, n = ints(torch, before), ints(torch, news)

    def step():
        p = g.kv_plan(b, n, free, tables, 16, 23)
        cache.store(k, k, p.slots)
        return (cache.attend(q, p.starts, p.lens, tables, max_new=20), *cache.load(p.slots))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    side = torch.cuda.Stream()
    for i in range(4):
        k.copy_(torch.randn(23, KV, D, device="cuda").bfloat16())
        for x in out:
            x.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), i


# --------------------------------------------------------------------------- #
# refusals
# --------------------------------------------------------------------------- #
def test_refusals(torch):
    cache, (k, kp, v, vp) = empty(torch, "mx4", 4, 2, 16, 64)
    e8, e4, e2 = torch.float8_e8m0fnu, torch.float8_e4m3fn, torch.float4_e2m1fn_x2
    with pytest.raises(ValueError, match="are needed"):
        g.KVCache(k.view(e2), v.view(e2))
    with pytest.raises(ValueError, match="are needed"):
        g.KVCache(k.view(e4), v.view(e4), kp.view(e8))
    with pytest.raises(TypeError, match="float8_e8m0fnu"):
        g.KVCache(k.view(e2), v.view(e2), kp, vp)
    with pytest.raises(ValueError, match="shape"):
        g.KVCache(k.view(e2), v.view(e2), kp[:3].view(e8), vp[:3].view(e8))
    with pytest.raises(ValueError, match="belong"):
        x = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
        g.KVCache(x, x.clone(), kp.view(e8), vp.view(e8))
    with pytest.raises(ValueError, match="multiple of 32"):
        g.KVCache(k[..., :24].view(e2), v[..., :24].view(e2), kp.view(e8), vp.view(e8))
    turned = kp.permute(2, 1, 0, 3).contiguous().permute(2, 1, 0, 3).view(e8)
    with pytest.raises(ValueError, match="strides"):
        g.KVCache(k.view(e2), v.view(e2), turned, vp.view(e8))
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        cache.load(slots, torch.float32)
    with pytest.raises(TypeError, match="slots"):
        cache.load(slots.int())
    with pytest.raises(ValueError, match="3 rows"):
        cache.load(slots, keys=torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError, match="3 rows"):
        cache.load(slots, torch.float16, values=torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda"))
    y = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(g.GorioError, match="overlap"):
        cache.load(slots, keys=y, values=y)
    assert cache.load(slots[:0])[0].shape == (0, 2, 64)
    plain = g.KVCache(*[torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)])
    with pytest.raises(g.GorioError, match="own type"):
        plain.load(slots, torch.float16)
