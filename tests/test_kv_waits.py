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
__global__ void largest(const u32x4 *a, float *out) { read(a, out, [](const f32x16 &s) { return max16<false>(s); }); }
__global__ void reciprocals(const float *a, float *out) {
  f32x16 s;
  for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_rcpf(a[threadIdx.x + 64 * i]);
  s[2] = __builtin_amdgcn_rcpf(s[2]);
  out[threadIdx.x] = max16<true>(s);
}
"""


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    """The kernels' instructions, by kernel."""
    at = tmp_path_factory.mktemp("waits")
    (at / "probe.hip").write_text(SOURCE)
    subprocess.run([_build.HIPCC, *_build.FLAGS, "-w", f"-I{_build.CSRC}", "--cuda-device-only", "-S", "-o",
                    str(at / "probe.s"), str(at / "probe.hip")], check=True, capture_output=True, timeout=300)
    found, name = {}, None
    for line in (at / "probe.s").read_text().splitlines():
        label = re.match(r"_Z\d+(plain|largest|reciprocals)\w*:", line)
        code = line.split(";")[0].strip()
        if label:
            name = label.group(1)
        elif name and code and not code.endswith(":") and not code.startswith("."):
            found.setdefault(name, []).append(code)
    return found


def registers(code):
    """Vector registers among an instruction's operands, the first written (as a rule), the others read."""
    return [int(r) for r in re.findall(r"\bv(\d+)\b", code.split(None, 1)[1] if " " in code else "")]


def product_to_read(code):
    """Wait states between the product and the first use of its result."""
    at = next(i for i, x in enumerate(code) if x.startswith("v_mfma"))
    first, last = map(int, re.search(r"v\[(\d+):(\d+)\]", code[at]).groups())
    states = 0
    for x in code[at + 1:]:
        if any(first <= r <= last for r in registers(x)):
            return states
        nop = re.match(r"s_nop (\d+)", x)
        states += int(nop.group(1)) + 1 if nop else 1
    raise AssertionError("the result is not used")


def test_the_largest_score_waits_for_the_product(assembly):
    plain = product_to_read(assembly["plain"])
    assert plain > 4                            # the compiler's own reads wait
    assert product_to_read(assembly["largest"]) >= plain


def test_the_largest_score_waits_for_reciprocals(assembly):
    code = [x for x in assembly["reciprocals"] if not x.startswith("s_waitcnt")]
    pairs = [(x, y) for x, y in zip(code, code[1:]) if x.startswith("v_rcp")]
    assert len(pairs) == 17
    for x, y in pairs:
        assert y.startswith(("v_rcp", "s_nop")) or registers(x)[0] not in registers(y)[1:], (x, y)
