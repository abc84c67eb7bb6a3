"""No touch of a matrix instruction's result before it is there, in the products and the attention of a decoding step: what the compiler made of a branch for each
scale converted one into a register that a 4-bit product ahead of the branch had still to write."""
import os
import subprocess

import pytest

from paper_2103_00130_amd import build as b
from test_around_step_build_cpu import early_touches

SOURCES = ["w4_bf16.hip", "w4_f16.hip", "w4_f32.hip", "kv_attention_bf16.hip", "kv_attention_f16.hip", "kv_attention_f32.hip"]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm")
    runs = {s: subprocess.Popen([b.HIPCC, *b.FLAGS, "-S", "--cuda-device-only", os.path.join(b.CSRC, s), "-o", str(out / s)], stderr=subprocess.DEVNULL) for s in SOURCES}
    assert not [s for s, r in runs.items() if r.wait() != 0]
    return {s: (out / s).read_text() for s in SOURCES}


@pytest.mark.parametrize("source", SOURCES)
def test_results_are_there_before_they_are_touched(assembly, source):
    # (a 16x16x64 product of bytes takes as long as the 16x16x32 ones of 16-bit types, whose states the search knows)
    text = assembly[source].replace("v_mfma_i32_16x16x64_i8", "v_mfma_i32_16x16x32_i8")
    assert "v_mfma" in text and not early_touches(text)
