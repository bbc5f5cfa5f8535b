"""Plain 64-bit forms of the paged key/value calls, one request, head and row at a time."""
import numpy as np


def attach(nodes, first_page, tokens, page, width, limit):
    B = len(nodes)
    tables, fills = np.full((B, width), -1, np.int32), np.full((B, width), page, np.int32)
    lens, attached = np.zeros(B, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        at = 0
        for v in nodes[b]:
            if v < 0 or v >= len(tokens):
                continue
            held = max(int(tokens[v]), 0)
            count = -(-held // page)
            if at + count > limit:
                break
            for i in range(count):
                tables[b, at + i] = first_page[v] + i
                fills[b, at + i] = min(page, held - i * page)
            at += count
            attached[b] += 1
        lens[b] = at * page
    return tables, fills, lens, attached


def plan(before, added, free, tables, page, T):
    tables = tables.copy()
    width = tables.shape[1]
    starts, lens, taken = [0], [], 0
    positions, slots = np.full(T, -1, np.int32), np.full(T, -1, np.int64)
    t = 0
    for b in range(len(before)):
        c, n = max(int(before[b]), 0), max(int(added[b]), 0)
        for e in range(min(-(-c // page), width), min(-(-(c + n) // page), width)):
            tables[b, e] = free[taken] if taken < len(free) else -1
            taken += 1
        for i in range(n):
            e = (c + i) // page
            if t < T:
                positions[t] = c + i
                if e < width and tables[b, e] >= 0:
                    slots[t] = int(tables[b, e]) * page + (c + i) % page
            t += 1
        starts.append(t)
        lens.append(c + n)
    return np.array(starts, np.int32), np.array(lens, np.int32), positions, slots, tables, taken


def visible(b, p, n_keys, a):
    """Keys that a token of request b at position p sees, by the definition."""
    page = a["page"]
    got = []
    for j in range(n_keys):
        e = j // page
        if e >= a["tables"].shape[1]:
            break
        if not 0 <= a["tables"][b, e] < len(a["keys"]):
            continue
        if a.get("fills") is not None and j % page >= a["fills"][b, e]:
            continue
        near = j <= p and (not a.get("window") or p - j < a["window"])
        if near or (a.get("prefix") is not None and j < a["prefix"][b]):
            got.append(j)
    return np.array(got, np.int64)


def attend(a):
    """(out, lse, bound): the attention in 64 bits, and how far a kernel with 32-bit sums
    may be from out at each element.

    u is half a step of out's type at 1 (2^-8 bf16, 2^-11 f16), A = sum_j w_j |v_j| / sum_j w_j:
      u |out|         the result's own rounding
      u A             each softmax weight is rounded to that type before the product
      4 e A           e = error of a score: it changes a weight by a factor of at most 1 + 2 e,
                      and the sum of the weights by as much.  e holds the dot product's D + 8
                      roundings to 24 bits of sum |q k| scale, the cap's tanh and the bias, each
                      to 2^-22 of its size, and 2^-19 for exp2 and the rescaling of partial sums
      2^-25 S / l     f16 only: weights below 2^-14 have steps of 2^-24; S = sum_j |v_j|, and
                      l = sum_j w_j is at least 1 where the largest weight is."""
    page, D = a["page"], a["D"]
    T, H = a["q"].shape[:2]
    G = H // a["keys"].shape[1]
    out, bound = np.zeros((T, H, D)), np.zeros((T, H, D))
    lse, lse_bound = np.full((T, H), -np.inf), np.zeros((T, H))
    u = 2.0 ** -8 if a["type"] == "bf16" else 2.0 ** -11
    for b in range(len(a["lens"])):
        t0, t1 = int(a["starts"][b]), int(a["starts"][b + 1])
        for t in range(t0, t1):
            p = int(a["lens"][b]) - (t1 - t0) + (t - t0)
            j = visible(b, p, int(a["lens"][b]), a)
            if not len(j):
                continue
            pages, place = a["tables"][b, j // page], j % page
            for h in range(H):
                k, v = a["keys"][pages, h // G, place], a["values"][pages, h // G, place]
                q = a["q"][t, h]
                s = a["scale"] * (k @ q)
                e = (D + 8) * 2.0 ** -24 * abs(a["scale"]) * (np.abs(k) @ np.abs(q)) + 2.0 ** -19
                if a.get("cap"):
                    s = a["cap"] * np.tanh(s / a["cap"])
                    e = e + 2.0 ** -22 * a["cap"]
                if a.get("slopes") is not None:
                    bias = a["slopes"][h] * np.abs(p - j)
                    s = s - bias
                    e = e + 2.0 ** -22 * np.abs(bias)
                e = e + 2.0 ** -22 * np.abs(s)
                m = s.max()
                if m == -np.inf:
                    continue
                w = np.exp(s - m)
                l = w.sum()
                out[t, h] = w @ v / l
                e = float(e[w > 0].max())
                A = w @ np.abs(v) / l
                bound[t, h] = u * np.abs(out[t, h]) + (u + 4 * e) * A
                if a["type"] == "f16":
                    bound[t, h] += 2.0 ** -25 * np.abs(v).sum(0) / l
                lse[t, h] = m + np.log(l)
                lse_bound[t, h] = 2 * e + 2.0 ** -22 * abs(lse[t, h])
    return out, lse, bound, lse_bound
