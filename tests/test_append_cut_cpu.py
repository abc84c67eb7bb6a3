"""Among how many tokens a workgroup of an append looks for runs: the sizes of the GPU tests reach every window."""
import ctypes
import os
import subprocess

import pytest

from test_gpu_rotary_runs import WINDOWS

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2103_00130_amd", "csrc")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("cut") / "cut.so")
    src = ('#include "kv_append_cut.h"\nextern "C" {\nint plain(long long tokens, int heads) { return abft::append_window(tokens, heads); }\n'
           'int rotary(long long tokens, int heads, int block) { return abft::rotary_window(tokens, heads, block); }\n'
           'int most() { return abft::kMaxWindow; }\n}\n')
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", "-x", "c++", "-", "-o", lib], input=src, text=True, check=True)
    so = ctypes.CDLL(lib)
    so.plain.argtypes, so.rotary.argtypes = [ctypes.c_longlong, ctypes.c_int], [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    return so


def test_windows_of_the_gpu_tests(rules):
    for _, heads, _, block, tokens, window in WINDOWS:
        assert rules.rotary(tokens, heads, block) == window, (heads, block, tokens)
    assert {w[-1] for w in WINDOWS} == {2, 4, 8, 16, 32, 64} and {w[3] for w in WINDOWS} == {16, 32, 64, 128}


def test_windows_are_no_wider_than_a_block_and_a_wavefront(rules):
    for block in (16, 32, 64, 128):
        for heads in (1, 2, 3, 16, 1000, 2 ** 31 - 1):
            for tokens in (1, 7, 300, 5000, 0xffffff):
                w = rules.rotary(tokens, heads, block)
                assert 1 <= w <= min(block, rules.most()) and w & (w - 1) == 0
                assert 1 <= rules.plain(tokens, heads) <= 16
