"""What the compiler makes of the kernels around a decoding step: no spilled registers, nothing ahead of the instruction that makes all lanes
active, and no touch of a matrix instruction's result before it is there.

The last: the compiler puts wait states between a matrix instruction and what reads or overwrites its result, but where several branches lead
there it counts along the first that it finds.  Sums of a loop were stored one instruction behind their last product, which was lost."""
import os
import re
import subprocess

import pytest

from paper_2103_00130_amd import build as b
from test_decode_build_cpu import early_vector_work

SOURCES = ["kv_rotary.hip", "lora.hip", "logprobs.hip"]


def registers(text):
    r = set()
    for kind, first, last in re.findall(r"\b([av])\[(\d+):(\d+)\]", text):
        r |= {(kind, k) for k in range(int(first), int(last) + 1)}
    return r | {(kind, int(k)) for kind, k in re.findall(r"\b([av])(\d+)\b", text)}


def early_touches(asm):
    """(kernel, matrix instruction, what touches its result, states between them) along every path; a 16x16x4 product of binary32 needs 10
    states, the 16x16x32 products of 16-bit types 8 (what the compiler puts between them within a block)."""
    lines = [x.split(";")[0].strip() for x in asm.split("\n")]
    labels = {x[:-1]: i for i, x in enumerate(lines) if re.match(r"\.LBB\S+:$", x)}
    kernel, found = None, []
    for i, line in enumerate(lines):
        if re.match(r"_Z\S+:$", line):
            kernel = line[:-1]
        if not line.startswith("v_mfma"):
            continue
        op, rest = line.split(None, 1)
        result, needed = registers(rest.split(",")[0]), 10 if op.endswith("16x16x4_f32") else 8 if "16x16x32" in op else None
        assert needed, f"{op}: how many states?"
        paths, seen = [(i + 1, 0)], set()
        while paths:
            at, states = paths.pop()
            while states < needed and at < len(lines):
                x = lines[at]
                if re.match(r"_Z\S+:$", x) or x.startswith("s_endpgm"):
                    break
                at += 1
                if not x or x.startswith(".") or x.endswith(":"):
                    continue
                name, *operands = x.split(None, 1)
                operands = operands[0] if operands else ""
                states += int(operands) + 1 if name == "s_nop" else 1
                if name == "s_branch" or name.startswith("s_cbranch"):
                    to = (labels[operands], states)
                    if to not in seen:
                        seen.add(to)
                        paths.append(to)
                    if name == "s_branch":
                        break
                elif name.startswith("v_mfma"):
                    into, *factors = operands.split(",")
                    if registers(",".join(factors[:2])) & result:
                        found.append((kernel, line, x, states - 1))
                    if result <= registers(into):
                        break       # (a sum that goes on: the matrix cores keep its order)
                elif registers(operands) & result:
                    found.append((kernel, line, x, states - 1))
                    break
    return found


def test_the_search_finds_what_it_looks_for():
    loop = "_Zk:\n.LBB0_1:\n\tv_mfma_f32_16x16x4_f32 a[0:3], v0, v1, a[0:3]\n\ts_cbranch_scc0 .LBB0_1\n.LBB0_2:\n\tWAIT\n\tds_write_b128 v9, a[0:3]\n\ts_endpgm\n"
    assert early_touches(loop.replace("WAIT", "s_nop 7")) == [("_Zk", "v_mfma_f32_16x16x4_f32 a[0:3], v0, v1, a[0:3]", "ds_write_b128 v9, a[0:3]", 9)]
    assert not early_touches(loop.replace("WAIT", "s_nop 8"))
    assert early_touches("_Zk:\n\tv_mfma_f32_16x16x32_f16 v[0:3], v[4:7], v[8:11], 0\n\ts_nop 6\n\tv_mov_b32_e32 v2, 0\n") and not early_touches(
        "_Zk:\n\tv_mfma_f32_16x16x32_f16 v[0:3], v[4:7], v[8:11], 0\n\ts_nop 7\n\tv_mov_b32_e32 v2, 0\n")


def test_no_vote_inside_a_choice():
    """A ballot on one side of `c ? a : b` is taken by the lanes that come to that side alone.  Such a vote, for the rows that the lanes on the
    other side had, found none, and the row that was read instead lay ahead of the first."""
    def votes(text):
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)
        return [s.strip() for s in re.split(r"[;{}]", text) if "?" in s and re.search(r"__ballot|__any|__all|__shfl|readlane", s.split("?", 1)[1])]
    assert votes("{ const int m = on ? lane : __builtin_ctz(__ballot(on)); }") and votes("x = on ? __shfl(a, 1) : 0;")
    assert not votes("const auto r = __ballot(on); // ? __ballot\n const int m = on ? lane : __builtin_ctz(r); a = __ballot(b ? c : d) ")
    for name in ("kv_append.h", *SOURCES):
        found = votes(open(os.path.join(b.CSRC, name)).read())
        assert not found, (name, found)


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm")
    runs = {s: subprocess.Popen([b.HIPCC, *b.FLAGS, "-S", "--cuda-device-only", os.path.join(b.CSRC, s), "-o", str(out / s)], stderr=subprocess.DEVNULL) for s in SOURCES}
    assert not [s for s, r in runs.items() if r.wait() != 0]
    return {s: (out / s).read_text() for s in SOURCES}


@pytest.mark.parametrize("source", SOURCES)
def test_kernels(assembly, source):
    spills = re.findall(r"\.vgpr_spill_count:\s*(\d+)", assembly[source])
    assert spills and set(spills) == {"0"}
    # (nor private memory: a function that is not inlined has the kernel's parameters copied there)
    assert set(re.findall(r"\.private_segment_fixed_size:\s*(\d+)", assembly[source])) == {"0"}
    assert not early_vector_work(assembly[source])
    assert not early_touches(assembly[source])
    assert source != "lora.hip" or "v_mfma" in assembly[source]
