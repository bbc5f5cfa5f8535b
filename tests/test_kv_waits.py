"""Registers that a matrix instruction writes are not read before it is done.

The compiler places the wait states for reads that it knows of, and none for
those of inline assembly.  The attention kernels' assembly that takes a
product's result is compiled right behind the product, and has to wait as long
as a plain read does (runs without a GPU).
"""
import re
import subprocess

import pytest

from paper_2607_04415_amd import _build

SOURCE = """
#include "kv_attend.hpp"
using namespace gorio;
template <typename F>
__device__ void read(const u32x4 *a, float *out, F f) {
  f32x16 s;
  for (int i = 0; i < 16; ++i) s[i] = 0.f;
  s = KvBf16::mfma32(a[threadIdx.x], a[threadIdx.x + 64], s);
  out[threadIdx.x] = f(s);
}
__global__ void plain(const u32x4 *a, float *out) { read(a, out, [](const f32x16 &s) { return s[0] + s[1]; }); }
__global__ void largest(const u32x4 *a, float *out) { read(a, out, [](const f32x16 &s) { return max16(s); }); }
"""


@pytest.fixture(scope="module")
def waits(tmp_path_factory):
    """Wait states between the product and the first read of its result, by kernel."""
    at = tmp_path_factory.mktemp("waits")
    (at / "probe.hip").write_text(SOURCE)
    subprocess.run([_build.HIPCC, *_build.FLAGS, "-w", f"-I{_build.CSRC}", "--cuda-device-only", "-S", "-o",
                    str(at / "probe.s"), str(at / "probe.hip")], check=True, capture_output=True, timeout=300)
    found, name, states, written = {}, None, None, range(0)
    for line in (at / "probe.s").read_text().splitlines():
        label = re.match(r"_Z\d+(plain|largest)\w*:", line)
        if label:
            name, states = label.group(1), None
            continue
        code = line.split(";")[0].strip()
        if not code or code.endswith(":") or code.startswith(".") or name is None:
            continue
        product = re.match(r"v_mfma_\w+ v\[(\d+):(\d+)\]", code)
        if product:
            written, states = range(int(product.group(1)), int(product.group(2)) + 1), 0
        elif states is not None and name not in found:
            operands = code.split(None, 1)[1] if " " in code else ""
            if any(int(r) in written for r in re.findall(r"\bv(\d+)\b", operands)):
                found[name] = states
            nop = re.match(r"s_nop (\d+)", code)
            states += int(nop.group(1)) + 1 if nop else 1
    return found


def test_the_largest_score_waits_for_the_product(waits):
    assert waits["plain"] > 4                   # the compiler's own reads wait
    assert waits["largest"] >= waits["plain"]
