"""The workspace of a call with groups: by the sizes, and with a window by whether there is a prefix (runs without a GPU)."""
import ctypes

import pytest

import paper_2607_04415_amd as g
from paper_2607_04415_amd import kv
from test_kv_args import attention, cache, lib, workspace  # noqa: F401


def need(lib, **more):  # noqa: F811
    c, a = cache(dtype=kv.MX4), attention(requests=5, tokens=7, width=1 << 20, **more)
    n, s = ctypes.c_uint64(), kv.SharingDesc(groups=2)
    assert lib.gorio_kv_workspace_shared(ctypes.byref(c), ctypes.byref(a), ctypes.byref(s), ctypes.byref(n)) == g.OK
    return n.value, workspace(lib, c, a)[1]


@pytest.mark.parametrize("window", [0, 1, 300])
def test_workspace_goes_by_sizes_and_a_prefix(lib, window):  # noqa: F811
    """Addresses that nothing is at: none is read."""
    plain = need(lib)[1]
    with_sums = need(lib)[0]
    assert with_sums >= plain + 7 * 4 * 66 * 4
    assert need(lib, window=window, prefix=64) == (with_sums, plain)
    assert need(lib, window=window) == (plain if window else with_sums, plain)
    for more in (dict(fills=64), dict(slopes=64), dict(q=64, out=64, lse=64), dict(starts=64, lens=64, tables=64), dict(cap=20.0)):
        assert need(lib, window=window, prefix=64, **more) == (with_sums, plain)
