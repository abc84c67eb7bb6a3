"""What the compiler makes of the kernels of a decoding step, in two ways in which it went wrong without a word.

A matrix instruction's result is not touched before it is there: of a branch for each scale it had made a conversion into a register that a 4-bit
product ahead of the branch had still to write.

No vector instruction stands where no lane is active: behind a loop that runs until none is, or where a branch leads that is taken when none
is, ahead of what makes lanes active again.  A copy that stood there, of a constant that the loop had put aside, was made by no lane, where more than 256 registers
were in use; the search in test_decode_build_cpu ends at the next label, behind which the lanes came back."""
import os
import re
import subprocess

import pytest

from paper_2103_00130_amd import build as b
from test_around_step_build_cpu import early_touches

PRODUCTS = ["w4_bf16.hip", "w4_f16.hip", "w4_f32.hip", "kv_attention_bf16.hip", "kv_attention_f16.hip", "kv_attention_f32.hip"]
OTHERS = ["kv_rotary.hip", "kv_cache.hip", "kv_plan.hip", "logprobs.hip", "lora.hip"]


def idle_vector_work(asm):
    """(kernel, instruction) that would be executed by no lane."""
    lines = [x.split(";")[0].strip() for x in asm.split("\n")]
    lines = [x for x in lines if x and (not x.startswith(".") or re.match(r"\.LBB\S+:$", x))]
    labels = {x[:-1]: i for i, x in enumerate(lines) if x.startswith(".LBB")}
    fewer = r"s_\w+_saveexec|s_(and|andn2|xor)_b64 exec"
    kernel, starts, found = None, [], set()
    for i, x in enumerate(lines):
        if re.match(r"_Z\S+:$", x):
            kernel = x[:-1]
        branch = re.match(r"s_cbranch_exec(n?)z (\.LBB\S+)", x)
        if branch:
            # (only where lanes were just taken away: any other such branch is there for the shape of the code, and never or always taken)
            j = i - 1
            while not re.match(fewer, lines[j]) and not re.search(r":$|^s_cbranch|\bexec, exec\b", lines[j]):
                j -= 1
            if re.match(fewer, lines[j]):
                starts.append((kernel, i + 1 if branch.group(1) else labels[branch.group(2)]))
    for kernel, at in starts:
        for x in lines[at:]:
            if re.match(r"s_(c?branch|endpgm)|_Z", x) or re.search(r"\bexec\b", x.split(",")[0]) or "_saveexec" in x:
                break
            if re.match(r"v_(?!readlane|writelane|readfirstlane|nop)|global_|ds_|buffer_|flat_", x):
                found.add((kernel, x))
    return sorted(found)


def test_the_search_finds_what_it_looks_for():
    loop = ("_Zk:\n\ts_and_saveexec_b64 s[26:27], s[20:21]\n\ts_cbranch_execz .LBB0_75\n; %bb.1:\n\tv_mov_b32_e32 v160, 0xff\n\ts_and_b64 exec, exec, vcc\n"
            "\ts_cbranch_execz .LBB0_74\n.LBB0_73:\n\tv_add_u32_e32 v152, 64, v152\n\ts_andn2_b64 exec, exec, s[28:29]\n\ts_cbranch_execnz .LBB0_73\n"
            ".LBB0_74:\n\tv_mov_b32_e32 v152, v160\n\ts_waitcnt vmcnt(0)\n.LBB0_75:\n\ts_or_b64 exec, exec, s[26:27]\n\tv_mov_b32_e32 v1, 0\n\ts_endpgm\n")
    assert idle_vector_work(loop) == [("_Zk", "v_mov_b32_e32 v152, v160")]
    assert not idle_vector_work(loop.replace("\tv_mov_b32_e32 v152, v160\n", ""))
    # a branch that stands for one that is always taken
    assert not idle_vector_work("_Zk:\n\ts_or_b64 exec, exec, s[6:7]\n\ts_cbranch_execnz .LBB0_2\n.LBB0_1:\n\tv_mov_b32_e32 v1, 0\n.LBB0_2:\n\ts_endpgm\n")


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm")
    runs = {s: subprocess.Popen([b.HIPCC, *b.FLAGS, "-S", "--cuda-device-only", os.path.join(b.CSRC, s), "-o", str(out / s)], stderr=subprocess.DEVNULL) for s in PRODUCTS + OTHERS}
    assert not [s for s, r in runs.items() if r.wait() != 0]
    return {s: (out / s).read_text() for s in PRODUCTS + OTHERS}


@pytest.mark.parametrize("source", PRODUCTS)
def test_results_are_there_before_they_are_touched(assembly, source):
    # (a 16x16x64 product of bytes takes as long as the 16x16x32 ones of 16-bit types, whose states the search knows)
    text = assembly[source].replace("v_mfma_i32_16x16x64_i8", "v_mfma_i32_16x16x32_i8")
    assert "v_mfma" in text and not early_touches(text)


@pytest.mark.parametrize("source", PRODUCTS + OTHERS)
def test_no_vector_work_without_lanes(assembly, source):
    assert "s_cbranch_exec" in assembly[source] and not idle_vector_work(assembly[source])


def test_rotated_appends_have_no_copies_in_other_registers(assembly):
    # (beyond 256 what is put aside goes to the registers of the matrix cores, by copies)
    counts = [int(n) for n in re.findall(r"\.vgpr_count:\s*(\d+)", assembly["kv_rotary.hip"])]
    assert counts and max(counts) <= 256
