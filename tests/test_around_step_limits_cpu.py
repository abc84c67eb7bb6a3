"""The largest and smallest calls of the operators around a decoding step, as the host sees them: what no launch can hold is refused as such."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2103_00130_amd", "csrc")


@pytest.fixture(scope="module")
def b():
    from paper_2103_00130_amd import binding
    return binding


def logprobs(b, rows=3, vocab=100, scale=1.0):
    d = ctypes.c_void_p(0x1000)
    return b.lib.abft_logprobs(d, vocab, 2, rows, vocab, scale, d, d, d, d, d, 0, None, None, None, 0, None)


def test_rows_of_logits_beyond_a_launch(b):
    # 2^24 workgroups of 256 threads are 2^32 threads
    for rows in (2 ** 24, 2 ** 24 + 1, 2 ** 31 - 1, 2 ** 31, 2 ** 40):
        assert logprobs(b, rows=rows) == b.ABFT_EUNSUPPORTED and b"too large" in b.lib.abft_last_error(), rows
        assert b.lib.abft_logprobs_workspace_bytes(rows, 100000, 5) == 0
    assert b.lib.abft_logprobs_workspace_bytes(2 ** 24 - 1, 100000, 5) > 0


def test_scales_under_which_differences_that_32_bits_do_not_hold_would_count(b):
    for scale in (2.0 ** -121, 1e-38, 2.0 ** -140):
        assert logprobs(b, scale=scale) == b.ABFT_EINVAL and b"scale" in b.lib.abft_last_error(), scale
    assert logprobs(b, rows=0, scale=2.0 ** -120) == b.ABFT_OK


def test_an_adapter_of_any_size_is_loaded_by_one_launch(tmp_path):
    src = '#include "lora_cut.h"\nextern "C" long long groups(long long elements) { return abft::lora_load_groups(elements); }\n'
    lib = str(tmp_path / "cut.so")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", "-x", "c++", "-", "-o", lib], input=src, text=True, check=True)
    f = ctypes.CDLL(lib).groups
    f.restype, f.argtypes = ctypes.c_longlong, [ctypes.c_longlong]
    assert [f(n) for n in (0, 1, 256, 257)] == [1, 1, 1, 2]
    for n in (2 ** 32 - 256, 2 ** 32 - 255, 2 ** 32, 2 ** 33, 128 * 2 * (2 ** 31 - 256)):
        assert 0 < f(n) * 256 < 2 ** 32, n


def test_sizes_of_more_than_32_bits_are_not_cut_to_them(b):
    for bad in ((2 ** 32 + 2, 64, 64, 8), (2, 2 ** 32 + 64, 64, 8), (2, 64, 2 ** 32 + 64, 8), (2, 64, 64, 2 ** 32 + 8)):
        with pytest.raises(ValueError):
            b.LoraPool(*bad, device="cpu")
    for bad in ((1, 2 ** 32 + 100000, 5), (1, 100000, 2 ** 32 + 5)):
        with pytest.raises(ValueError):
            b.abft_logprobs_workspace_bytes(*bad)

    class Pool:
        ref = ctypes.byref(b.abft_lora_t(0x1000, 0x1000, 0x1000, 0x1000, 3, 20, 100, 70, 2))
    with pytest.raises(ValueError):
        b.abft_lora_workspace_bytes(Pool, 2 ** 32 + 5)
    with pytest.raises(ValueError):
        b.abft_lora_load(Pool, 2 ** 32, None, None)
