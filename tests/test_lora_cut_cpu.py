"""How products with adapters are cut: the sizes of the GPU tests reach the form for prompts, and several blocks of columns to a wavefront."""
import ctypes
import os
import subprocess

import pytest

from test_gpu_lora_prompts import PROMPTS

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2103_00130_amd", "csrc")


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("cut") / "cut.so")
    src = ('#include "lora_cut.h"\nextern "C" void cut(long long M, int K, int N, int rank, int f32, int* out) {\n'
           '    const abft::LoraCut c = abft::lora_cut(M, K);\n    const int blocks = (N + abft::kLoraColumns - 1) / abft::kLoraColumns;\n'
           '    const int groups = abft::lora_up_groups(c, blocks, (rank + 15) / 16, f32), waves = groups * abft::kLoraWaves;\n'
           '    out[0] = c.tiles; out[1] = c.slots; out[2] = c.splits; out[3] = groups; out[4] = (blocks + waves - 1) / waves;\n}\n')
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", "-x", "c++", "-", "-o", lib], input=src, text=True, check=True)
    f = ctypes.CDLL(lib).cut
    f.argtypes = [ctypes.c_longlong] + [ctypes.c_int] * 4 + [ctypes.c_void_p]

    def of(M, K, N, rank, f32):
        out = (ctypes.c_int * 5)()
        f(M, K, N, rank, f32, out)
        return list(out)
    return of


def test_the_gpu_tests_reach_the_form_for_prompts(cut):
    slots, splits, ranks, wrong = set(), set(), set(), []
    for M, K, N, _, rank, blocks16, blocks32 in PROMPTS:
        for f32, blocks in ((0, blocks16), (1, blocks32)):
            c = cut(M, K, N, rank, f32)
            if c[4] != blocks:
                wrong.append((M, K, N, rank, f32, c))
            slots.add(c[1])
            splits.add(c[2])
            ranks.add((rank + 15) // 16)
    assert not wrong
    assert slots == {1, 8, 16} and {1, 3, 5} <= splits and ranks == {1, 2, 3, 4, 8}


def test_every_block_of_columns_has_a_wavefront(cut):
    for M in (1, 15, 16, 127, 300, 512, 5000, 16 * 65535):
        for N in (1, 64, 65, 4096, 100001, 2 ** 31 - 256):
            for rank in (1, 32, 33, 128):
                for f32 in (0, 1):
                    tiles, slots, _, groups, each = cut(M, 4096, N, rank, f32)
                    blocks = -(-N // 64)
                    assert groups >= 1 and each >= 1 and groups * 4 * each >= blocks and tiles <= 65535 and slots <= 16, (M, N, rank, f32)
