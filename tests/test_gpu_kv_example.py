"""The example program: search, tables, plans, stores and attention, one after the other."""
import importlib.util
from pathlib import Path

import numpy as np
import pytest

import kv_reference as ref

pytestmark = pytest.mark.gpu


def test_answer_from_passages():
    import torch
    path = Path(__file__).resolve().parents[1] / "examples" / "answer_from_passages.py"
    spec = importlib.util.spec_from_file_location("answer_from_passages", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.run(nodes=600, questions=3, found=4, answer=3)
    assert [len(y) for y in r["outputs"][1:]] == [3] * 3
    assert all(torch.isfinite(y.float()).all() for y in r["outputs"])
    # the last step's attention from the pages, in 64 bits
    host = lambda x: x.cpu().numpy()
    a = {"page": example.PAGE, "D": example.D, "type": "bf16", "scale": example.D ** -0.5, "window": 0, "cap": 0.0,
         "tables": host(r["tables"]), "fills": host(r["fills"]), "prefix": host(r["prefix"]), "lens": host(r["lens"]),
         "starts": host(r["starts"]), "q": host(r["q"].double()), "keys": host(r["cache"].keys.double()),
         "values": host(r["cache"].values.double())}
    out, _, bound, _ = ref.attend(a)
    assert (np.abs(host(r["out"].double()) - out) <= bound).all()
    assert (a["prefix"] > 0).all() and (a["lens"] > a["prefix"]).all()
