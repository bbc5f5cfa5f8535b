"""A row's powers begin at any byte: the compiler is told so where they are loaded (runs without a GPU)."""
import re
import subprocess

import pytest

from paper_2607_04415_amd import _build

SOURCE = """
#include "kv_attend_few.hpp"
using namespace gorio;
extern "C" __global__ void powers(uint64_t from, uint32_t count, Type *out) { *out = load_powers<kBlocks, Type>(from, count); }
"""


@pytest.mark.parametrize("blocks,type", [(2, "uint32_t"), (4, "uint32_t"), (6, "u32x2"), (8, "u32x2")])
def test_loads_of_powers_are_of_any_alignment(tmp_path, blocks, type):
    src, out = tmp_path / "powers.hip", tmp_path / "powers.ll"
    src.write_text(SOURCE.replace("kBlocks", str(blocks)).replace("Type", type))
    subprocess.run([_build.HIPCC, *_build.FLAGS, f"-I{_build.CSRC}", "--cuda-device-only", "-S", "-emit-llvm", "-o", str(out),
                    str(src)], check=True, capture_output=True)
    loads = re.findall(r"= load (?:\w+), ptr addrspace\(1\) %\w+(.*)", out.read_text())
    assert len(loads) == 2 and all(re.match(r", align 1\b", x) for x in loads), loads
