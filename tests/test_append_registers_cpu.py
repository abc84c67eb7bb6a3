"""Registers of the appends' kernels: as many wavefronts to a SIMD as the sizes of their units allow.  A loop over what a lane holds, unrolled too late, once doubled
the registers of all of them and took a quarter of their speed where prompts keep the chip half busy."""
import os
import re
import subprocess

import pytest

from paper_2103_00130_amd import build as b


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "kv_cache.s"
    subprocess.run([b.HIPCC, *b.FLAGS, "-S", "--cuda-device-only", os.path.join(b.CSRC, "kv_cache.hip"), "-o", str(out)], check=True, stderr=subprocess.DEVNULL)
    found = {}
    for entry in re.split(r"\n  - \.agpr_count", out.read_text())[1:]:
        name, count = re.search(r"\.name:\s+(\S+)", entry).group(1), int(re.search(r"\.vgpr_count:\s+(\d+)", entry).group(1))
        m = re.search(r"kv_append_kernelI(f|DF16_|DF16b)Lb([01])ELi(\d+)E", name)
        if m:
            found[m.group(1), m.group(2) == "1", int(m.group(3))] = count
    return found


# what a unit of U tokens of 8 columns holds is 4 U registers (8 U in binary32); four, five, six and eight wavefronts fit 128, 96, 80 and 64 registers
@pytest.mark.parametrize("unit,half,full", [(4, 64, 96), (8, 80, 128), (16, 128, 192)])
def test_registers_of_appends(kernels, unit, half, full):
    assert kernels["DF16b", True, unit] <= half and kernels["DF16_", True, unit] <= half and kernels["f", True, unit] <= full
