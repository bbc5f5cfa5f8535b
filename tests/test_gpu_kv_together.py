"""Search, tables, groups, plans, stores, attention and loads together, as a program that answers each
question several times over runs them."""
import importlib.util
from pathlib import Path

import numpy as np
import pytest

import kv_reference as ref
import mx_reference as mx
import paper_2607_04415_amd as g

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = Path(__file__).resolve().parents[1] / "examples" / "answer_from_passages.py"
    spec = importlib.util.spec_from_file_location("answer_from_passages", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


@pytest.mark.parametrize("pages,answers", [("mx4", 3), ("bf16", 2), ("mx4", 1)])
def test_answers_of_a_batch(example, pages, answers):
    import torch
    r = example.run(nodes=600, questions=3, found=4, answer=3, pages=pages, answers=answers)
    assert [len(y) for y in r["outputs"][1:]] == [3 * answers] * 3
    host = lambda x: x.cpu().numpy()
    cache = r["cache"]
    if pages == "mx4":
        values = [mx.unpack(host(x.view(torch.uint8)), host(s.view(torch.uint8)), "mx4")
                  for x, s in ((cache.keys, cache.key_scale), (cache.values, cache.value_scale))]
    else:
        values = [host(x.double()) for x in (cache.keys, cache.values)]
    a = {"page": example.PAGE, "D": example.D, "type": "bf16", "scale": example.D ** -0.5, "window": 0, "cap": 0.0,
         "tables": host(r["tables"]), "fills": host(r["fills"]), "prefix": host(r["prefix"]), "lens": host(r["lens"]),
         "starts": host(r["starts"]), "q": host(r["q"].double()), "keys": values[0], "values": values[1]}
    want, _, bound, _ = ref.attend(a)
    assert (np.abs(host(r["out"].double()) - want) <= bound).all()
    # the rows that the last step stored
    for got, x in zip(cache.load(r["slots"]), values):
        rows = x.swapaxes(1, 2).reshape(-1, example.KV_HEADS, example.D)[host(r["slots"])]
        assert np.array_equal(host(got.double()), rows)
    if answers == 1:
        assert r["sharing"] is None
        return
    # a question's answers share its passages, and the same by groups, in tables with room for them
    assert host(r["sharing"].first)[:4].tolist() == [0, answers, 2 * answers, 3 * answers]
    assert host(r["sharing"].shared).tolist() == [p if p >= 64 else 0 for p in host(r["prefix"])]
    room = torch.full((3 * answers, 20_000), -1, dtype=torch.int32, device="cuda")
    fills = torch.full_like(room, example.PAGE)
    room[:, :r["tables"].shape[1]], fills[:, :r["tables"].shape[1]] = r["tables"], r["fills"]
    out = cache.attend(r["q"], r["starts"], r["lens"], room, fills=fills, prefix=r["prefix"], sharing=r["sharing"])
    assert (np.abs(host(out.double()) - want) <= bound).all()
    again = g.kv_share(room, r["prefix"], example.PAGE, fills=fills, least=64)
    assert torch.equal(again.first, r["sharing"].first) and torch.equal(again.shared, r["sharing"].shared)
