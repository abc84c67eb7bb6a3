"""What the compiler makes of the attention kernels, whose registers are nearly all in use.

A kernel that spilled vector registers faulted: the copy of a spilled address stood between the label that a divergent branch jumps to
and the instruction that makes all lanes active again, so that no lane made it.  So no kernel may spill, and no join of a divergent
branch may hold vector work ahead of that instruction."""
import os
import re
import subprocess

import pytest

from paper_2103_00130_amd import build as b


def early_vector_work(asm):
    """(kernel, instruction) where a join of a divergent branch writes vector registers before all lanes are active."""
    lines = asm.split("\n")
    joins = {m.group(1) for line in lines for m in [re.search(r"s_cbranch_execz (\.LBB\S+)", line)] if m}
    kernel, found = None, []
    for i, line in enumerate(lines):
        m = re.match(r"(_Z\S+):", line)
        if m:
            kernel = m.group(1)
        m = re.match(r"(\.LBB\S+):", line)
        if not m or m.group(1) not in joins:
            continue
        ahead = []
        for t in (x.strip() for x in lines[i + 1:]):
            if re.match(r"\.LBB|s_cbranch|s_branch|s_and_saveexec|s_endpgm", t):
                break
            if re.match(r"s_or_b64 exec, exec|s_or_saveexec|s_mov_b64 exec", t):
                found += [(kernel, x) for x in ahead if re.match(r"v_(?!readlane|writelane)|global_|ds_|buffer_", x)]
                break
            ahead.append(t)
    return found


def test_the_search_finds_what_it_looks_for():
    bad = "_Zk:\n\ts_cbranch_execz .LBB0_2\n; %bb.1:\n\tv_mov_b32 v1, 0\n.LBB0_2:\n\tv_accvgpr_write_b32 a132, v86\n\ts_or_b64 exec, exec, s[0:1]\n"
    assert early_vector_work(bad) == [("_Zk", "v_accvgpr_write_b32 a132, v86")]
    assert not early_vector_work(bad.replace("\tv_accvgpr_write_b32 a132, v86\n", ""))


SOURCES = ["kv_attention_f32.hip", "kv_attention_f16.hip", "kv_attention_bf16.hip", "kv_cache.hip", "w4_f32.hip", "w4_f16.hip", "w4_bf16.hip", "kv_plan.hip"]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm")
    runs = {s: subprocess.Popen([b.HIPCC, *b.FLAGS, "-S", "--cuda-device-only", os.path.join(b.CSRC, s), "-o", str(out / s)], stderr=subprocess.DEVNULL) for s in SOURCES}
    assert not [s for s, r in runs.items() if r.wait() != 0]
    return {s: (out / s).read_text() for s in SOURCES}


@pytest.mark.parametrize("source", SOURCES)
def test_kernels_do_not_spill(assembly, source):
    spills = re.findall(r"\.vgpr_spill_count:\s*(\d+)", assembly[source])
    assert spills and set(spills) == {"0"}
    assert not early_vector_work(assembly[source])
