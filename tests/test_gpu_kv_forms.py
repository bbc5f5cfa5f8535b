"""Which form takes a request goes by its own rows: what stands beside it in a batch does not change its bits."""
import numpy as np
import pytest

import paper_2607_04415_amd as g
from test_gpu_kv import call, ints
from test_gpu_kv_shared import ROOM, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def first_of(torch, a, n, groups):
    """The call's first n requests alone."""
    more = {} if groups is None else {"sharing": g.KVSharing(ints(torch, groups), ints(torch, a["shared"][:n]))}
    t = int(a["starts"][n])
    return call(torch, {**a, "tables": a["tables"][:n], "lens": a["lens"][:n], "starts": a["starts"][:n + 1]},
                q=a["q_gpu"][:t], **more)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3"), ("bf16", "mx4"), ("f16", "mx8")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shared", [0, 64])
def test_single_tokens_beside_a_prompt(torch, type, cache, D, shared):
    """Single tokens of up to 500 keys of their own, which the form for few rows does not divide, and 64 shared
    ones, which are one block: with a prompt of 600 behind them they are computed as without it."""
    page, KV = 16, 2
    width = ROOM // (2 * KV * D * page * 5) + 1
    a = inputs(torch, D, type, cache, 4, KV, D, page, [5, 1], [1, 1, 2, 1, 1, 600], [500, 40, 333, 7, 129, 610], [shared, 0],
               width=width, poison=False)
    groups = [0, 5, 6] if shared else None
    want = first_of(torch, a, 5, [0, 5] if shared else None)
    got = first_of(torch, a, 6, groups)
    for x, y in zip(got, want):
        assert torch.equal(x[:6], y)
    assert np.isfinite(got[0].float().cpu().numpy()).all()
