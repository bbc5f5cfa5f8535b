"""Scores under caps of every size, on the GPU against the formula in 64 bits."""
import numpy as np
import pytest

import kv_reference as ref
from test_gpu_kv import call, setup, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def attend(a):
    """(out, lse, bound, lse bound) as kv_reference.attend has them, but for the cap's part of a
    score's error: 2^-15 up to a cap of 64 and 2^-20 of the capped score past that, as stated."""
    T, H = a["q"].shape[:2]
    G, page, D = H // a["keys"].shape[1], a["page"], a["D"]
    out, bound, lse, lse_bound = np.zeros((T, H, D)), np.zeros((T, H, D)), np.zeros((T, H)), np.zeros((T, H))
    u = 2.0 ** -11
    for b in range(len(a["lens"])):
        t0, t1 = a["starts"][b], a["starts"][b + 1]
        for t in range(t0, t1):
            p = int(a["lens"][b] - t1 + t)
            j = ref.visible(b, p, int(a["lens"][b]), a)
            pages, place = a["tables"][b, j // page], j % page
            for h in range(H):
                k, v, q = a["keys"][pages, h // G, place], a["values"][pages, h // G, place], a["q"][t, h]
                s = a["scale"] * (k @ q)
                e = (D + 8) * 2.0 ** -24 * abs(a["scale"]) * (np.abs(k) @ np.abs(q)) + 2.0 ** -19
                s = a["cap"] * np.tanh(s / a["cap"])
                e = e + (2.0 ** -15 if a["cap"] <= 64 else 2.0 ** -20 * np.abs(s))
                if a.get("slopes") is not None:
                    bias = a["slopes"][h] * np.abs(p - j)
                    s, e = s - bias, e + 2.0 ** -22 * np.abs(bias)
                e = e + 2.0 ** -22 * np.abs(s)
                w = np.exp(s - s.max())
                l, e = w.sum(), float(e[w > 0].max())
                out[t, h] = w @ v / l
                bound[t, h] = (u * np.abs(out[t, h]) + (u + 4 * e) * (w @ np.abs(v)) / l
                               + 2.0 ** -25 * np.abs(v).sum(0) / l)
                lse[t, h] = s.max() + np.log(l)
                lse_bound[t, h] = 2 * e + 2.0 ** -22 * abs(lse[t, h])
    return out, lse, bound, lse_bound


@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("news,D", [([1, 4], 64), ([50, 30], 64), ([2, 3], 200), ([40], 96), ([40], 128), ([30], 200)])
@pytest.mark.parametrize("cap,spread", [(50.0, 6.0), (64.0, 1.0), (65.0, 6.0), (300.0, 6.0), (3000.0, 1.0), (3e4, 6.0),
                                        (1e6, 1.0), (1e8, 6.0), (1e38, 1.0)])
def test_caps(torch, cap, spread, news, D, slopes):  # noqa: F811
    """Scores far below the cap, beside it and past it: none is lost in the cap's size."""
    a = setup(torch, 29, "f16", "f16", 4, 2, D, 16, news, [150, 130][:len(news)], cap=cap, spread=spread, slopes=slopes)
    out, lse = (x.double().cpu().numpy() for x in call(torch, a))
    w_out, w_lse, bound, lse_bound = attend(a)
    assert (np.abs(lse - w_lse) <= lse_bound).all(), np.abs(lse - w_lse).max()
    assert (np.abs(out - w_out) <= bound).all(), np.abs(out - w_out).max()


@pytest.mark.parametrize("news", [[1, 4], [50, 30]])
@pytest.mark.parametrize("cap,scale", [(1e-42, 0.125), (1e-42, -0.125), (1e-3, 1e37)])
def test_caps_of_no_size(torch, cap, scale, news):  # noqa: F811
    """scale / cap passes float32: scores are 0 or the cap, and products of 0 stay 0."""
    a = setup(torch, 31, "f16", "f16", 4, 2, 64, 16, news, [150, 130], cap=cap, scale=scale)
    a["q_gpu"][::2] = 0
    a["q"][::2] = 0
    a["cap"] = cap
    out, lse = (x.double().cpu().numpy() for x in call(torch, a))
    w_out, w_lse, bound, _ = attend({**a, "scale": min(abs(scale), 1.0) * np.sign(scale)})
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    few = 2.0 ** -15
    assert (np.abs(lse - w_lse) <= few).all() and (np.abs(out - w_out) <= bound + few * np.abs(a["values"]).max()).all()
