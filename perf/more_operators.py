"""Performance cases of small key/value pages and of shared prefixes, and their plain forms.

A program that answers from passages keeps their attention keys and values in
pages in HBM.  A case is one of five operators on such pages:

  store   new keys and values -> pages of 8 or 4 bits, each 32 elements of a row
          with a power of two of their own; the pages are then read back whole;
  load    rows of such pages at given slots -> 16-bit values;
  attend  attention of new tokens over such pages;
  share   request tables -> groups of requests whose first pages are the same;
  joint   attention of a batch in which each group's first pages are the same.

Pages of type "mx8" hold e4m3 values, "mx4" e2m1 values, two a byte, the element
with the even index in the low half.  32 elements x of a row share 2^E, kept as
the byte E + 127: E is the smallest number in -127..127 with max |x| <= 448 * 2^E
(6 * 2^E for mx4), and 255 stands for a block that holds a NaN or an infinity,
all of which then reads as NaN.  An element is x / 2^E, rounded to the nearest,
halves to even, and stands for its value times 2^E.

Virtual position j of request b is place j % page of the page that entry
j // page of row b of the table names.  A head h of the queries reads key and
value head h // (heads / kv).  Key j is visible to a new token at position p if
its place is below the page's fill, j < lens[b], and (j <= p and p - j < window,
or j < prefix[b]).  The score is scale * q.k, then cap * tanh(score / cap) where a
cap is set.  A row without a visible key gives 0, and -inf as its log-sum-exp.

Two neighbouring requests share c positions: the page's tokens times the number
of leading entries in which their rows, and the fills, are equal, but at most the
whole pages that each holds.  A request joins the group of the one before it if
c >= least; a group shares the smallest c of its neighbours, a single request 0.

Sizes are those of the repository's own workloads (1M nodes, k = 10, rows of 128
and 96 elements, pages of 16 tokens) and generic ones around them.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
MOST = {"mx8": 448.0, "mx4": 6.0, "e4m3": 448.0}
BLOCK = 32                                    # elements with a scale of their own
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# --------------------------------------------------------------------------- #
# the cases
# --------------------------------------------------------------------------- #
def _store(tokens, heads, kv, D, page, type, cache):
    return {"op": "store", "tokens": tokens, "heads": heads, "kv": kv, "D": D, "page": page, "type": type,
            "cache": cache}


def _load(tokens, held, kv, D, page, type, cache):
    return {"op": "load", "tokens": tokens, "held": held, "kv": kv, "D": D, "page": page, "type": type, "cache": cache}


def _share(requests, width, groups, page, fills=False):
    return {"op": "share", "requests": requests, "width": width, "groups": groups, "page": page, "fills": fills}


def _attend(requests, new, context, heads, kv, D, page=16, type="bf16", cache="mx4", ragged=True, passages=False,
            cap=0.0, window=0, lse=False, shared=0, groups=1):
    return {"op": "joint" if shared else "attend", "requests": requests, "new": new, "context": context,
            "heads": heads, "kv": kv, "D": D, "page": page, "type": type, "cache": cache, "ragged": ragged,
            "passages": passages, "cap": cap, "window": window, "lse": lse, "shared": shared, "groups": groups}


def listed():
    return [
        # one decoding step's keys and values: all latency
        dict(_store(64, 32, 8, 128, 16, "bf16", "mx4"), name="store-step-mx4"),
        # a long prompt's keys and values, rows of 96
        dict(_store(16384, 24, 4, 96, 24, "f16", "mx8"), name="store-prompt-mx8"),
        # the ten passages of one search, moved to another cache
        dict(_load(2000, 100_000, 8, 128, 16, "bf16", "mx4"), name="load-passages-mx4"),
        # a long text read back in one go
        dict(_load(16384, 20_000, 8, 128, 16, "f16", "mx8"), name="load-prompt-mx8"),
        # one decoding step of a serving batch: which requests have a prompt in common
        dict(_share(64, 1060, 5, 16), name="share-step"),
        # a batch of questions, many of which found the same passages
        dict(_share(1000, 512, 90, 16, fills=True), name="share-1000"),
        # one user's answer, token by token over a thousand tokens
        dict(_attend(1, 1, 1000, 32, 8, 128, cache="mx4"), name="attend-one-mx4"),
        # one decoding step of a serving batch over long texts
        dict(_attend(64, 1, 16384, 32, 8, 128, cache="mx4"), name="attend-step-mx4"),
        # questions of some hundred tokens over the passages found for them, heads of 96, scores capped
        dict(_attend(4, 500, 8192, 24, 4, 96, type="f16", cache="mx8", passages=True, cap=50.0, lse=True),
             name="attend-questions-mx8"),
        # eight answers to one question, token by token
        dict(_attend(8, 1, 300, 32, 8, 128, cache="mx4", shared=2000), name="joint-samples-mx4"),
        # one decoding step of a batch that works on the same long text
        dict(_attend(64, 1, 500, 32, 8, 128, cache="bf16", shared=16384, lse=True), name="joint-step"),
        # questions of some ten tokens, each group about the same passages
        dict(_attend(100, 40, 400, 32, 8, 128, type="f16", cache="e4m3", passages=True, shared=8000, groups=3),
             name="joint-questions-e4m3"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "load", "share", "attend", "attend", "joint", "joint"])
    type = rng.choice(["bf16", "f16"])
    kv = rng.choice([1, 2, 4, 8])
    D = rng.choice([64, 96, 128, 128, 160])
    page = rng.choice([8, 16, 16, 24, 64])
    if op == "store":
        return _store(_log(rng, 1, 16384), kv * rng.choice([1, 4, 6]), kv, D, page, type, rng.choice(["mx8", "mx4"]))
    if op == "load":
        held = _log(rng, 100, 100_000)
        return _load(_log(rng, 1, 16384), held, kv, D, page, type, rng.choice(["mx8", "mx4"]))
    if op == "share":
        requests = _log(rng, 8, 1000)
        return _share(requests, _log(rng, 64, 1100), rng.randint(1, requests // 3), page, rng.random() < 0.5)
    new = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 500)])
    case = _attend(_log(rng, 1, 128), new, 0, kv * rng.choice([1, 2, 4, 5, 8]), kv, D, page=page, type=type,
                   cache=rng.choice(["mx8", "mx4"]), ragged=rng.random() < 0.7, passages=rng.random() < 0.4,
                   cap=rng.choice([0.0, 0.0, 30.0]), window=rng.choice([0, 0, 0, rng.randint(1, 4096)]),
                   lse=rng.random() < 0.5)
    if op == "attend":
        case["context"] = case["new"] + _log(rng, 1, 16384)
    else:
        case.update(op="joint", context=case["new"] + _log(rng, 1, 1000), shared=_log(rng, 16, 16384),
                    cache=rng.choice(["mx8", "mx4", "e4m3", type, type]), window=0)
        case["requests"] = max(2, case["requests"])
        case["groups"] = rng.randint(1, max(1, min(4, case["requests"] // 2)))
    most = 0.9 * work(listed()[-1])["flops"]
    while work(case)["flops"] > most or case["requests"] * _context(case) * case["kv"] * D > 6.5e8:
        if case["requests"] > 2 * case["groups"]:
            case["requests"] = max(2 * case["groups"], (case["requests"] + 1) // 2)
        elif case["shared"] > 32:
            case["shared"] = (case["shared"] + 1) // 2
        else:
            case["context"] = (case["context"] + 1) // 2
            case["new"] = min(case["new"], case["context"])
    return case


def _context(case):
    return case["context"] + case["shared"]


def _pairs_at_most(case):
    return case["requests"] * case["new"] * _context(case) * case["heads"] * case["D"]


# --------------------------------------------------------------------------- #
# small pages
# --------------------------------------------------------------------------- #
def _pack(x, cache):
    """Rows of float values -> (elements, scale bytes) of pages of this type."""
    x = x.unflatten(-1, (-1, BLOCK))
    most = x.abs().amax(-1, keepdim=True).float()                      # NaN where there is one
    m, e = torch.frexp(most)
    e = e - (8 if cache == "mx8" else 2) - 1 + (m * 2 > MOST[cache] / (256 if cache == "mx8" else 4)).int()
    e = torch.where(most == 0, -127, e).clamp(-127, 127)
    bad = ~torch.isfinite(most)
    u = x.double() * torch.exp2(-e.double())
    u = torch.where(bad, 0.0, u)
    scale = torch.where(bad, 255, e + 127).to(torch.uint8)[..., 0]
    u = u.flatten(-2)
    if cache == "mx8":
        return u.float().to(torch.float8_e4m3fn).view(torch.uint8), scale   # exact in float
    step = torch.exp2(torch.frexp(u.abs().clamp(min=1.0)).exponent.double() - 2)
    size = torch.round(u.abs() / step) * step
    at = torch.bucketize(size.float(), torch.tensor(E2M1, device=u.device)).int()
    code = (at + 8 * torch.signbit(u).int()).to(torch.uint8)
    return code[..., ::2] | (code[..., 1::2] << 4), scale


def _unpack(elements, scale, cache):
    """(elements, scale bytes) -> the values they stand for, in 32 bits."""
    if cache == "mx8":
        x = elements.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=elements.device)
        x = table[torch.stack((elements & 15, elements >> 4), -1).flatten(-2).int()]
    s = torch.exp2(scale.double() - 127)
    s = torch.where(scale == 255, math.nan, s)
    return (x.unflatten(-1, (-1, BLOCK)) * s[..., None]).float().flatten(-2)


def _small(case):
    return case["cache"] in ("mx8", "mx4")


def _cache(case, pages):
    """An empty cache as the program keeps it: [page][kv head][token][element]."""
    shape, D = (pages, case["kv"], case["page"]), case["D"]
    s = {"key_scale": None, "value_scale": None}
    for name in ("key", "value"):
        if _small(case):
            s[name + "s"] = torch.zeros((*shape, D // 2 if case["cache"] == "mx4" else D), dtype=torch.uint8, device=DEV)
            s[name + "_scale"] = torch.zeros((*shape, D // BLOCK), dtype=torch.uint8, device=DEV)
        elif case["cache"] == "e4m3":
            s[name + "s"] = torch.zeros((*shape, D), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
            s[name + "_scale"] = torch.tensor([(0.013 if name == "key" else 0.009) * (1 + 0.11 * h)
                                               for h in range(case["kv"])], dtype=torch.float32, device=DEV)
        else:
            s[name + "s"] = torch.zeros((*shape, D), dtype=TYPES[case["cache"]], device=DEV)
    if own:
        import paper_2607_04415_amd as g
        kept = [s[n] for n in ("keys", "values", "key_scale", "value_scale")]
        if _small(case):
            kind = torch.float8_e4m3fn if case["cache"] == "mx8" else torch.float4_e2m1fn_x2
            kept = [x.view(kind) for x in kept[:2]] + [x.view(torch.float8_e8m0fnu) for x in kept[2:]]
        s["cache"] = g.KVCache(*kept)
    return s


def _fill(case, s, gen, pages):
    """Keys and values of earlier tokens; keys lean to one side, as trained ones do."""
    kv, D = case["kv"], case["D"]
    lean = 0.7 * torch.randn((kv, 1, D), generator=gen, device=DEV)
    for name in ("key", "value"):
        for lo in range(0, pages, 4096):
            part = s[name + "s"][lo:lo + 4096]
            x = torch.randn((len(part), kv, case["page"], D), generator=gen, device=DEV)
            x = x + lean if name == "key" else x
            if _small(case):
                part.copy_(_pack(x, case["cache"])[0])
                s[name + "_scale"][lo:lo + 4096] = _pack(x, case["cache"])[1]
            elif case["cache"] == "e4m3":
                part.copy_((x / s[name + "_scale"][:, None, None]).clamp_(-448, 448).to(part.dtype))
            else:
                part.copy_(x.to(part.dtype))


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _group_of(case):
    """Each request's group: neighbours, of sizes that differ by at most one."""
    return np.arange(case["requests"]) * case["groups"] // case["requests"]


def _shared(case):
    """What each request shares with its group: whole pages, the first group the most."""
    if not case["shared"]:
        return np.zeros(case["requests"], np.int64)
    g = _group_of(case)
    pages = max(1, case["shared"] // case["page"])
    return np.maximum(1, (pages * (1 - 0.21 * g / case["groups"])).astype(np.int64)) * case["page"]


def _lengths(case):
    """New tokens and all tokens of each request: the first has the most of both.
    Ragged batches spread them, and one of their requests has nothing new."""
    r = random.Random("%d %d %d" % (case["requests"], case["new"], case["context"]))
    new, total = [case["new"]], [case["context"]]
    for b in range(1, case["requests"]):
        if case["ragged"]:
            n = 0 if b == 5 else max(1, _log(r, max(1, case["new"] // 16), case["new"]))
            t = max(n, int(r.uniform(0.25, 1.0) * case["context"]))
        else:
            n, t = case["new"], case["context"]
        new.append(n)
        total.append(t)
    return np.array(new), np.array(total) + _shared(case)


def _prefix(case):
    """The passages' positions: all of what is shared, or all that is whole pages before the new tokens."""
    if not case["passages"]:
        return np.zeros(case["requests"], np.int64)
    new, total = _lengths(case)
    return _shared(case) if case["shared"] else (total - new) // case["page"] * case["page"]


def _fills(case, entries):
    """Tokens held by each table entry of a prefix of passages: each eighth page ends a passage."""
    e = np.arange(entries)
    return np.where(e % 8 == 7, 1 + (5 * e) % case["page"], case["page"])


def _ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def _normal(shape, type, gen, spread=1.0):
    return torch.randn(shape, generator=gen, device=DEV).mul_(spread).to(type)


def _prepare_store(case, gen):
    page, T = case["page"], case["tokens"]
    pages = -(-T // page) + 1
    s = _cache(case, pages)
    # the rows of a fused projection: queries, then keys, then values; heads of different sizes
    rows = torch.randn((T, case["heads"] + 2 * case["kv"], case["D"]), generator=gen, device=DEV)
    rows *= torch.exp2(torch.randn((1, rows.shape[1], 1), generator=gen, device=DEV) * 2)
    order = torch.randperm(pages, generator=gen, device=DEV)
    j = torch.arange(T, device=DEV) + int(torch.randint(0, page, (1,), generator=gen, device=DEV))
    slots = order[(j // page) % pages] * page + j % page
    slots[torch.rand(T, generator=gen, device=DEV) < 0.01] = -1             # padding
    s.update(rows=rows.to(TYPES[case["type"]]), slots=slots, all=torch.arange(pages * page, device=DEV))
    return s


def _prepare_load(case, gen):
    page, T = case["page"], case["tokens"]
    pages = -(-case["held"] // page)
    s = _cache(case, pages)
    _fill(case, s, gen, pages)
    # runs of up to 200 tokens, each from the first place of some page
    run = torch.randint(0, pages, (T // 200 + 1,), generator=gen, device=DEV)
    t = torch.arange(T, device=DEV)
    slots = (run[t // 200] + t % 200 // page) % pages * page + t % 200 % page
    slots[torch.rand(T, generator=gen, device=DEV) < 0.01] = -1
    s.update(slots=slots)
    return s


def _prepare_share(case, gen):
    B, width, page = case["requests"], case["width"], case["page"]
    # each request's own pages, over the first of which its group's are laid
    tables = torch.randperm(B * width, generator=gen, device=DEV).int().reshape(B, width)
    g = torch.randint(0, case["groups"], (B,), generator=gen, device=DEV).sort().values
    common = torch.randint(width // 4, width, (case["groups"],), generator=gen, device=DEV)[g]
    e = torch.arange(width, device=DEV)
    tables = torch.where(e < common[:, None], tables[g] + B * width, tables).contiguous()
    held = common * page + torch.randint(0, 40 * page, (B,), generator=gen, device=DEV)
    tables[e >= ((held + page) // page)[:, None]] = -1
    s = {"tables": tables, "held": held.int(), "fills": None, "least": 128}
    if case["fills"]:
        s["fills"] = torch.where(e % 8 == 7, 1 + (5 * e) % page, page).int().expand(B, width).contiguous()
    return s


def _prepare_attend(case, gen):
    new, total = _lengths(case)
    page, kv, D = case["page"], case["kv"], case["D"]
    shared = _shared(case)
    entries, common = -(-total // page), shared // page
    width, own_pages = int(entries.max()), int((entries - common).sum())
    g = _group_of(case)
    first = np.concatenate([[0], np.nonzero(np.diff(g))[0] + 1])
    all_pages = own_pages + int(common[first].sum()) + 3
    s = _cache(case, all_pages)
    _fill(case, s, gen, all_pages)
    order = torch.randperm(all_pages, generator=gen, device=DEV).int()
    e = torch.arange(width, device=DEV)
    tables = torch.full((len(new), width), -1, dtype=torch.int32, device=DEV)
    tables[(e >= _ints(common)[:, None]) & (e < _ints(entries)[:, None])] = order[:own_pages]
    at = own_pages + np.concatenate([[0], np.cumsum(common[first])])
    start = _ints(at[:-1][g] if case["shared"] else np.zeros(len(new)))
    tables = torch.where(e < _ints(common)[:, None], order[(start[:, None] + e).clamp(max=all_pages - 1)], tables)
    T = int(new.sum())
    s.update(q=_normal((T, case["heads"], D), TYPES[case["type"]], gen, 1.2), tables=tables.contiguous(), T=T,
             width=width, lens=_ints(total), starts=_ints(np.concatenate([[0], np.cumsum(new)])), fills=None,
             prefix=None, sharing=None, most_new=int(new.max()), scale=D ** -0.5)
    if case["passages"]:
        prefix = _prefix(case)
        s["prefix"] = _ints(prefix)
        held = np.full((len(new), width), page)
        for b in range(len(new)):
            held[b, : prefix[b] // page] = _fills(case, prefix[b] // page)
        s["fills"] = _ints(held)
    if case["shared"]:
        s["first"], s["shared"] = _ints(np.concatenate([first, [len(new)]])), _ints(shared)
        if own:
            import paper_2607_04415_amd as g_
            s["sharing"] = g_.KVSharing(s["first"], s["shared"])
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"store": _prepare_store, "load": _prepare_load, "share": _prepare_share, "attend": _prepare_attend,
         "joint": _prepare_attend}[case["op"]](case, gen)
    s["case"] = case
    return s


# --------------------------------------------------------------------------- #
# the plain forms
# --------------------------------------------------------------------------- #
def _plain_store(s):
    case = s["case"]
    page, kv, slots, type = case["page"], case["kv"], s["slots"], TYPES[case["type"]]
    at = (slots >= 0).nonzero()[:, 0]
    p, o = slots[at] // page, slots[at] % page

    def put(name, lo):
        elements, scale = _pack(s["rows"][:, lo:lo + kv][at], case["cache"])
        s[name + "s"][p, :, o] = elements
        s[name + "_scale"][p, :, o] = scale
        x = _unpack(s[name + "s"], s[name + "_scale"], case["cache"])
        return x.permute(0, 2, 1, 3).reshape(-1, kv, case["D"]).to(type)

    return {"keys": put("key", case["heads"]), "values": put("value", case["heads"] + kv)}


def _plain_load(s):
    case = s["case"]
    page, slots = case["page"], s["slots"]
    p, o = slots.clamp(min=0) // page, slots.clamp(min=0) % page

    def get(name):
        x = _unpack(s[name + "s"][p, :, o], s[name + "_scale"][p, :, o], case["cache"])
        return torch.where(slots[:, None, None] >= 0, x, 0.0).to(TYPES[case["type"]])

    return {"keys": get("key"), "values": get("value")}


def _plain_share(s):
    case = s["case"]
    page, B, tables, held = case["page"], case["requests"], s["tables"], s["held"].long()
    same = tables[1:] == tables[:-1]
    if s["fills"] is not None:
        same = same & (s["fills"][1:] == s["fills"][:-1])
    common = same.long().cumprod(1).sum(1)
    common = torch.minimum(common, torch.minimum(held[1:], held[:-1]) // page) * page
    joins = common >= s["least"]
    begins = torch.cat([joins.new_ones(1), ~joins])
    group = begins.long().cumsum(0) - 1
    b = torch.arange(B, device=DEV)
    first = torch.full((B + 1,), B, device=DEV).scatter_reduce(0, group, b, "amin")
    none = 1 << 40
    least = torch.full((B,), none, device=DEV).scatter_reduce(0, group[1:], torch.where(joins, common, none), "amin")
    shared = least[group]
    return {"first": first.int(), "shared": torch.where(shared == none, 0, shared).int()}


def _plain_attend(s):
    case = s["case"]
    page, kv, D, heads = case["page"], case["kv"], case["D"], case["heads"]
    B, width, N, T = case["requests"], s["width"], s["most_new"], s["T"]
    L, G = width * page, heads // kv
    at = s["tables"].long().clamp(min=0)

    def rows(name):
        x, scale = s[name + "s"][at], s[name + "_scale"]
        if _small(case):
            x = _unpack(x, scale[at], case["cache"])
        x = x.permute(0, 2, 1, 3, 4).reshape(B, kv, L, D).float()
        return x.mul_(scale[:, None, None]) if case["cache"] == "e4m3" else x

    starts, lens = s["starts"].long(), s["lens"].long()
    new = starts[1:] - starts[:-1]
    n = torch.arange(N, device=DEV)
    t = (starts[:-1, None] + n).clamp(max=T - 1)
    q = s["q"][t].float().reshape(B, N, kv, G, D).permute(0, 2, 3, 1, 4).reshape(B, kv, G * N, D)
    x = torch.matmul(q, rows("key").transpose(2, 3).contiguous()).mul_(s["scale"]).reshape(B, kv, G, N, L)
    if case["cap"] > 0:
        x = x.div_(case["cap"]).tanh_().mul_(case["cap"])
    p = ((lens - new)[:, None] + n)[:, :, None]                       # B, N, 1
    j = torch.arange(L, device=DEV)[None, None, :]
    seen = j <= p
    if case["window"] > 0:
        seen = seen & (p - j < case["window"])
    if s["prefix"] is not None:
        seen = seen | (j < s["prefix"].long()[:, None, None])
    there = (s["tables"] >= 0).repeat_interleave(page, 1) & (j[0] < lens[:, None])
    if s["fills"] is not None:
        there = there & (j[0] % page < s["fills"].repeat_interleave(page, 1))
    x.masked_fill_(~(seen & there[:, None, :])[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    lse = m + total.log()
    o = torch.matmul(x.reshape(B, kv, G * N, L), rows("value")).reshape(B, kv, G, N, D)
    o = torch.where(total > 0, o / total, 0.0)
    b = torch.searchsorted(starts, torch.arange(T, device=DEV), right=True) - 1
    i = torch.arange(T, device=DEV) - starts[b]
    out = {"out": o.permute(0, 3, 1, 2, 4)[b, i].reshape(T, heads, D).to(s["q"].dtype)}
    if case["lse"]:
        out["lse"] = lse[..., 0].permute(0, 3, 1, 2)[b, i].reshape(T, heads)
    return out


# --------------------------------------------------------------------------- #
# one pass
# --------------------------------------------------------------------------- #
def _own_store(s):
    c = s["case"]
    s["cache"].store(s["rows"][:, -2 * c["kv"]:-c["kv"]], s["rows"][:, -c["kv"]:], s["slots"])
    keys, values = s["cache"].load(s["all"], TYPES[c["type"]])
    return {"keys": keys, "values": values}


def _own_load(s):
    keys, values = s["cache"].load(s["slots"], TYPES[s["case"]["type"]])
    return {"keys": keys, "values": values}


def _own_share(s):
    import paper_2607_04415_amd as g
    got = g.kv_share(s["tables"], s["held"], s["case"]["page"], fills=s["fills"], least=s["least"])
    return {"first": got.first, "shared": got.shared}


def _own_attend(s):
    c = s["case"]
    got = s["cache"].attend(s["q"], s["starts"], s["lens"], s["tables"], fills=s["fills"], prefix=s["prefix"],
                            scale=s["scale"], cap=c["cap"], window=c["window"], max_new=s["most_new"],
                            with_lse=c["lse"], sharing=s["sharing"])
    return {"out": got[0], "lse": got[1]} if c["lse"] else {"out": got}


def run(state):
    forms = ((_own_store, _own_load, _own_share, _own_attend, _own_attend) if own else
             (_plain_store, _plain_load, _plain_share, _plain_attend, _plain_attend))
    return dict(zip(("store", "load", "share", "attend", "joint"), forms))[state["case"]["op"]](state)


# --------------------------------------------------------------------------- #
# what a pass cannot do without
# --------------------------------------------------------------------------- #
def _visible(case):
    """(row, key) pairs of one head, and the keys that some row sees, a group's shared ones once."""
    new, total = _lengths(case)
    prefixes, shared, group = _prefix(case), _shared(case), _group_of(case)
    page, pairs, keys = case["page"], 0, 0
    window = case["window"] or (1 << 40)
    for b, (n, t, prefix) in enumerate(zip(new.tolist(), total.tolist(), prefixes.tolist())):
        there = np.ones(t, np.int64)
        if prefix:
            there[:prefix] = (np.arange(page) < _fills(case, prefix // page)[:, None]).reshape(-1)
        upto = np.concatenate([[0], np.cumsum(there)])
        p = np.arange(t - n, t)
        left = np.maximum(0, p + 1 - window)
        pairs += int((upto[p + 1] - upto[np.maximum(left, np.minimum(prefix, p + 1))] + upto[prefix]).sum())
        if n:
            keys += int(upto[t] - upto[max(prefix, int(left[0]))] + upto[prefix])
        if shared[b]:                                                  # no windows here: all see them
            keys -= int(upto[shared[b]]) if n else 0
            keys += int(upto[shared[b]]) if b == 0 or group[b] != group[b - 1] else 0
    return pairs, keys


def _row_bytes(case):
    D = case["D"]
    return case["kv"] * {"mx4": D / 2 + D / BLOCK, "mx8": D + D / BLOCK, "e4m3": D}.get(case["cache"], 2 * D)


def work(case):
    if case["op"] == "store":
        rows, pages = case["tokens"], (-(-case["tokens"] // case["page"]) + 1) * case["page"]
        wide = 2 * case["kv"] * case["D"]
        return {"bytes": 8 * rows + 2 * rows * (wide + _row_bytes(case)) + 2 * pages * (wide + _row_bytes(case)) + 8 * pages,
                "flops": 0}
    if case["op"] == "load":
        return {"bytes": case["tokens"] * (8 + 2 * (2 * case["kv"] * case["D"] + _row_bytes(case))), "flops": 0}
    if case["op"] == "share":
        # up to where two rows differ: five eighths of a row, as these are made
        return {"bytes": case["requests"] * (2.5 * case["width"] * (2 if case["fills"] else 1) + 12), "flops": 0}
    pairs, keys = _visible(case)
    T = int(_lengths(case)[0].sum())
    return {"bytes": 2 * keys * _row_bytes(case) + 4 * keys // case["page"] + 4 * T * case["heads"] * case["D"]
            + (4 * T * case["heads"] if case["lse"] else 0),
            "flops": 4 * pairs * case["heads"] * case["D"]}


# --------------------------------------------------------------------------- #
# the same from the definitions, in 64 bits
# --------------------------------------------------------------------------- #
def _stands_for(s, name, at):
    """Values of cache rows in 64 bits; `at` indexes pages, heads and places."""
    case = s["case"]
    x, scale = s[name + "s"][at], s[name + "_scale"]
    if case["cache"] == "e4m3":
        head = at[1]
        return x.double() * scale.double()[head].reshape(-1, *[1] * (x.dim() - 1) if torch.is_tensor(head) else (1,))
    if not _small(case):
        return x.double()
    power = scale[at].double() - 127
    power[scale[at] == 255] = math.nan
    if case["cache"] == "mx4":
        x = torch.stack([x % 16, x // 16], -1).reshape(*x.shape[:-1], -1)
        sign, exponent, bit = x // 8, x % 8 // 2, x % 2
    else:
        sign, exponent, bit = x // 128, x % 128 // 8, x % 8
    bits, bias = (1, 1) if case["cache"] == "mx4" else (3, 7)
    size = torch.where(exponent == 0, bit.double() * 2.0 ** (1 - bias - bits),
                       (1 + bit.double() * 2.0 ** -bits) * torch.exp2(exponent.double() - bias))
    return torch.where(sign == 1, -size, size) * torch.exp2(power).repeat_interleave(BLOCK, -1)


def _exact_store(s):
    c = s["case"]
    page, kv, D, out = c["page"], c["kv"], c["D"], {}
    bits, lowest, most = (3, -6, 448.0) if c["cache"] == "mx8" else (1, 0, 6.0)
    t = torch.nonzero(s["slots"] >= 0).reshape(-1)
    for name, lo in (("keys", c["heads"]), ("values", c["heads"] + kv)):
        x = s["rows"][t, lo:lo + kv].double().reshape(len(t), kv, D // BLOCK, BLOCK)
        biggest = x.abs().max(-1, keepdim=True).values
        power = torch.ceil(torch.log2(biggest / most))
        power = torch.where(biggest > most * torch.exp2(power), power + 1, power)      # log2 is not exact
        power = torch.where(biggest <= most * torch.exp2(power - 1), power - 1, power)
        power = power.clamp(-127, 127)
        u = x / torch.exp2(power)
        step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** lowest))) - bits)
        pages = len(s["keys"])
        flat = torch.zeros((pages * page, kv, D), dtype=torch.float64, device=DEV)
        flat[s["slots"][t]] = (torch.round(u / step) * step * torch.exp2(power)).reshape(len(t), kv, D)
        out[name] = flat
    return out


def _exact_load(s):
    page, slots = s["case"]["page"], s["slots"]
    out = {}
    for name in ("key", "value"):
        p, o = slots.clamp(min=0) // page, slots.clamp(min=0) % page
        x = _stands_for(s, name, (p[:, None], torch.arange(s["case"]["kv"], device=DEV)[None], o[:, None]))
        x[slots < 0] = 0
        out[name + "s"] = x
    return out


def _exact_share(s):
    c = s["case"]
    tables, held = s["tables"].cpu().numpy(), s["held"].cpu().numpy().astype(np.int64)
    fills = None if s["fills"] is None else s["fills"].cpu().numpy()
    first, shared, least = [0], [], []
    for b in range(1, c["requests"] + 1):
        got = 0
        if b < c["requests"]:
            differs = tables[b] != tables[b - 1]
            if fills is not None:
                differs |= fills[b] != fills[b - 1]
            got = int(np.argmax(differs)) if differs.any() else c["width"]
            got = min(got, int(held[b]) // c["page"], int(held[b - 1]) // c["page"]) * c["page"]
        if b < c["requests"] and got >= s["least"]:
            least.append(got)
        else:
            shared += [min(least, default=0)] * (b - first[-1])
            first.append(b)
            least = []
    first += [c["requests"]] * (c["requests"] + 1 - len(first))
    return {"first": _ints(first), "shared": _ints(shared)}


def _exact_attend(s):
    c = s["case"]
    page, kv, D, G = c["page"], c["kv"], c["D"], c["heads"] // c["kv"]
    new, total = _lengths(c)
    out = torch.zeros((s["T"], c["heads"], D), dtype=torch.float64, device=DEV)
    lse = torch.full((s["T"], c["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    t0 = 0
    for b, (n, t) in enumerate(zip(new.tolist(), total.tolist())):
        j = torch.arange(t, device=DEV)
        entry = s["tables"][b].long()[j // page]
        ok = torch.ones(t, dtype=torch.bool, device=DEV)
        if s["fills"] is not None:
            ok = j % page < s["fills"][b].long()[j // page]
        j, entry = j[ok], entry[ok]
        for h in range(kv):
            k, v = _stands_for(s, "key", (entry, h, j % page)), _stands_for(s, "value", (entry, h, j % page))
            k = k.t().contiguous()
            p = torch.arange(t - n, t, device=DEV)[:, None]
            mask = j <= p
            if c["window"]:
                mask &= j > p - c["window"]
            if s["prefix"] is not None:
                mask |= j < s["prefix"][b]
            for g in range(G):
                x = s["q"][t0:t0 + n, h * G + g].double() @ k * s["scale"]
                if c["cap"]:
                    x = torch.tanh(x / c["cap"]) * c["cap"]
                x = torch.where(mask, x, -math.inf)
                z = torch.logsumexp(x, 1)
                w = torch.exp(x - torch.where(z == -math.inf, 0.0, z)[:, None])
                out[t0:t0 + n, h * G + g] = w @ v
                lse[t0:t0 + n, h * G + g] = z
        t0 += n
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


def exact(case, seed):
    if case["op"] in ("attend", "joint") and (_pairs_at_most(case) > 6e11 or case["requests"] * case["heads"] > 20000):
        return None                                                    # over about 20 seconds
    return {"store": _exact_store, "load": _exact_load, "share": _exact_share, "attend": _exact_attend,
            "joint": _exact_attend}[case["op"]](prepare(case, seed))
