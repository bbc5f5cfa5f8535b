"""Answer from the passages that a search finds.

A small retrieval program on one GPU: nodes of an index stand for passages of
text, each with its attention keys and values kept in pages in HBM.  For a
batch of questions the program searches the index, makes each question's table
of pages from the ids found, writes the question's own keys and values into
pages of a free list, and attends to all of it: first the question at once,
then the answer token by token.  The "model" is one attention layer with random
weights; what a program with a trained one would change is where its queries,
keys and values come from.

Each question may be answered several times over.  Its answers read the same
passages, so their requests follow one another in the batch, and attention is
told which first pages they have in common.  Pages hold 16 bits an element, or 4
with a power of two for each 32.

    python examples/answer_from_passages.py [--pages mx4] [--answers 3]
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import numpy as np
import torch

ROOT = Path(__file__).resolve().parents[1]
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))

import paper_2607_04415_amd as g  # noqa: E402
from workload import IndexSpec, QuerySpec, index_arrays, query_array  # noqa: E402

HEADS, KV_HEADS, D, PAGE = 8, 2, 128, 16      # a 4 KB page of a head: 16 tokens of 128 16-bit values
HIDDEN = HEADS * D


class Layer:
    """Projections of one attention layer, random but seeded."""

    def __init__(self, seed: int):
        gen = torch.Generator().manual_seed(seed)
        rows = (HEADS + 2 * KV_HEADS) * D
        self.w = (torch.randn(HIDDEN, rows, generator=gen) / HIDDEN ** 0.5).bfloat16().cuda()
        self.out = (torch.randn(HEADS * D, HIDDEN, generator=gen) / (HEADS * D) ** 0.5).bfloat16().cuda()

    def project(self, x):
        rows = (x @ self.w).view(len(x), HEADS + 2 * KV_HEADS, D)
        return rows[:, :HEADS], rows[:, HEADS:-KV_HEADS], rows[:, -KV_HEADS:]


def empty_cache(pages: int, type: str) -> g.KVCache:
    shape = (pages, KV_HEADS, PAGE)
    if type == "bf16":
        return g.KVCache(*(torch.zeros((*shape, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    halves = [torch.zeros((*shape, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    powers = [torch.zeros((*shape, D // 32), dtype=torch.uint8, device="cuda") for _ in range(2)]
    return g.KVCache(*(x.view(torch.float4_e2m1fn_x2) for x in halves), *(x.view(torch.float8_e8m0fnu) for x in powers))


def run(nodes: int = 3000, questions: int = 4, found: int = 5, answer: int = 8, seed: int = 0, pages: str = "bf16",
        answers: int = 1) -> dict:
    rng = np.random.default_rng(seed)
    gen = torch.Generator().manual_seed(seed)
    text = lambda n: torch.randn(n, HIDDEN, generator=gen).bfloat16().cuda()   # embedded tokens
    layer = Layer(seed)

    # the index, and each node's passage: its tokens and the pages that hold them
    spec = IndexSpec(n=nodes, D=128, dtype="u8", clusters=8, sigma=20.0, r_near=16, r_rand=16, seed=31)
    arrays = index_arrays(spec, use_cache=False)
    index = g.Index(arrays["x"], arrays["graph"])
    tokens = rng.integers(5, 61, nodes).astype(np.int32)
    held = -(-tokens // PAGE)
    first_page = (np.cumsum(held) - held).astype(np.int32)
    spare = 256 * answers
    free = torch.arange(int(held.sum()), int(held.sum()) + spare, dtype=torch.int32, device="cuda")
    cache = empty_cache(int(held.sum()) + spare, pages)
    at = np.concatenate([f * PAGE + np.arange(t) for f, t in zip(first_page, tokens)])
    _, k, v = layer.project(text(int(tokens.sum())))
    cache.store(k, v, torch.from_numpy(at).cuda())

    # the questions: what the search finds becomes each one's prefix
    ids, _, _ = index.search(torch.from_numpy(query_array(spec, QuerySpec(questions, 7))).cuda(), k=found, L=32, W=4,
                             stats=False)
    ids = ids.repeat_interleave(answers, 0)          # a question's requests follow one another
    width = found * 4 + 16
    tables, fills, lens, _ = g.kv_attach(ids, torch.from_numpy(first_page).cuda(), torch.from_numpy(tokens).cuda(),
                                         PAGE, width, limit=found * 4)
    prefix = lens.clone()
    new = torch.from_numpy(rng.integers(3, 30, questions).astype(np.int32)).repeat_interleave(answers)
    outputs = []
    x = text(int(new.sum()))
    # what the requests have in common does not change from step to step: the passages
    sharing = g.kv_share(tables, lens, PAGE, fills=fills, least=64) if answers > 1 else None
    for step in range(1 + answer):
        plan = g.kv_plan(lens, new.cuda(), free, tables, PAGE, len(x))
        q, k, v = layer.project(x)
        cache.store(k, v, plan.slots)
        out = cache.attend(q, plan.starts, plan.lens, tables, fills=fills, prefix=prefix, max_new=int(new.max()),
                           sharing=sharing)
        y = out.reshape(len(x), HEADS * D) @ layer.out
        outputs.append(y)
        last = dict(q=q, starts=plan.starts, lens=plan.lens, out=out, slots=plan.slots, sharing=sharing)
        free, lens = free[int(plan.taken):], plan.lens
        # the next token of each answer comes from the last row of its request
        x = torch.nn.functional.normalize(y[(plan.starts[1:] - 1).long()].float(), dim=1).mul(HIDDEN ** 0.5).bfloat16()
        new = torch.ones(questions * answers, dtype=torch.int32)
    return dict(ids=ids, tables=tables, fills=fills, prefix=prefix, cache=cache, outputs=outputs, **last)


if __name__ == "__main__":
    args = argparse.ArgumentParser()
    args.add_argument("--pages", choices=("bf16", "mx4"), default="bf16")
    args.add_argument("--answers", type=int, default=1)
    r = run(**vars(args.parse_args()))
    torch.cuda.synchronize()
    print(f"{len(r['prefix'])} requests, {r['prefix'].tolist()} positions of passages, "
          f"{r['lens'].tolist()} in all after {len(r['outputs'])} steps")
