"""Values and keys that only some rows of a tile see, and tiles of every size, on the GPU."""
import numpy as np
import pytest

import kv_reference as ref
from test_gpu_kv import call, holds, setup, torch  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f16", "f16"), ("f16", "e4m3")]


@pytest.mark.parametrize("type,cache", TYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 200, 256])
@pytest.mark.parametrize("news,opts", [(3, {}), (100, {}), (100, dict(window=30)), (300, dict(cap=20.0)),
                                       (300, dict(window=90, slopes=True))])
def test_not_finite_where_some_rows_see_it(torch, type, cache, D, news, opts):  # noqa: F811
    """NaN and inf among the chunk's own tokens reach the rows that see them, at their element, and no other."""
    n, length = news, news + 70
    a = setup(torch, D + n, type, cache, 4, 2, D, 16, [n], [length], poison=False, **opts)
    at = length - n // 2                                # the first token's place that holds one
    low = D // 2 - 1
    odd = [(0, 3, "nan"), (1, low, "nan")]              # key head, element
    if cache != "e4m3":
        odd += [(1, D - 5, "inf"), (1, D - 1, "-inf"), (0, low, "inf"), (0, D // 2, "-inf")]
    pages = a["cache"].values.view(torch.uint8) if cache == "e4m3" else a["cache"].values
    for h, d, what in odd:
        pages[a["tables"][0, at // 16], h, at % 16, d] = 0x7F if cache == "e4m3" else float(what)
    last = length - 1                                   # the last row alone sees a NaN key of the first key head
    keys = a["cache"].keys.view(torch.uint8) if cache == "e4m3" else a["cache"].keys
    keys[a["tables"][0, last // 16], 0, last % 16, D - 2] = 0x7F if cache == "e4m3" else float("nan")
    out, lse = (x.double().cpu().numpy() for x in call(torch, a))
    w_out, w_lse, bound, lse_bound = ref.attend(a)
    p = length - n + np.arange(n)
    sees = (p >= at) & ((p - at < opts["window"]) if "window" in opts else True)
    hit = np.zeros(out.shape, bool)
    hit[-1, :2] = True
    assert np.isnan(out[-1, :2]).all() and np.isnan(lse[-1, :2]).all()
    for h, d, what in odd:
        rows = sees.copy()
        rows[-1] &= h != 0
        got = out[rows][:, 2 * h:2 * h + 2, d]
        assert np.isnan(got).all() if what == "nan" else np.array_equal(got, np.full_like(got, float(what)))
        hit[sees, 2 * h:2 * h + 2, d] = True
    assert (np.abs(out - w_out)[~hit] <= bound[~hit]).all()
    assert (np.abs(lse - w_lse)[:-1] <= lse_bound[:-1]).all()


@pytest.mark.parametrize("type,cache", TYPES)
@pytest.mark.parametrize("D,news", [(64, [150]), (96, [90, 70]), (128, [270]), (128, [140, 3, 150]), (200, [140]),
                                    (256, [140, 1])])
def test_several_tiles_of_a_request_cut(torch, type, cache, D, news):  # noqa: F811
    """Chunks of more rows than a tile has over texts long enough that their tiles are divided."""
    lens = [2000, 1500, 1700][:len(news)]
    a = setup(torch, D + len(news), type, cache, 2, 1, D, 16, news, lens, fills=True, prefix=[900] * len(news),
              window=400)
    holds(torch, a, call(torch, a))
