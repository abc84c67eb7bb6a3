"""What the binding and the library refuse, and how they cut their work, without a GPU."""
import ctypes
import os
import random
import subprocess

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2103_00130_amd import binding
    return binding


def test_memory_that_is_lent_is_contiguous_and_on_the_device(b):
    class OnDevice:      # (the questions that the binding asks of a tensor)
        is_cuda = True

        def __init__(self, t):
            self.t = t

        def __getattr__(self, name):
            return getattr(self.t, name)
    host = torch.empty(6)
    assert b._lent(None, "x") == (None, 0)
    assert b._lent(OnDevice(host), "x") == (host.data_ptr(), 24)
    with pytest.raises(TypeError):
        b._lent(host, "x")
    for t in (host[::2], host[:1].expand(6), host.reshape(2, 3).t()):
        with pytest.raises(ValueError):
            b._lent(OnDevice(t), "x")


def test_a_cache_of_the_host_is_refused(b):
    for device in ("cpu", torch.device("cpu"), "meta"):
        with pytest.raises(TypeError):
            b.KvCache(4, 2, 64, 16, device=device)


# --------------------------------------------------------------------------------------------- how attention is cut (csrc/kv_cut.h)
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2103_00130_amd", "csrc")
TOKENS, TOKENS8, ROWS = 0, 1, 2


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    """(columns, requests, heads, query heads for each, max_new, max_len) -> (kernel, workgroups for a request's rows, parts, tokens of a part)"""
    lib = str(tmp_path_factory.mktemp("cut") / "cut.so")
    src = ('#include "kv_cut.h"\nextern "C" void cut(int cols, int n, int heads, int group, int fresh, int len, int* out) {\n'
           '    const abft::AttnCut c = abft::attn_cut(cols, n, heads, group, fresh, len);\n    out[0] = c.shape; out[1] = c.groups; out[2] = c.parts; out[3] = c.chunk;\n}\n')
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", "-x", "c++", "-", "-o", lib],
                   input=src, text=True, check=True)
    so = ctypes.CDLL(lib)

    def call(*sizes):
        out = (ctypes.c_int * 4)()
        so.cut(*(ctypes.c_int(x) for x in sizes), out)
        return tuple(out)
    return call


# the sizes that the rule's comment has figures of, where one side is well ahead
@pytest.mark.parametrize("sizes,kernel,parts", [
    ((128, 1, 32, 1, 2000, 2000), ROWS, 1), ((64, 8, 16, 1, 1024, 1024), ROWS, 1), ((128, 2, 8, 5, 300, 6000), TOKENS, 1), ((64, 4, 12, 1, 512, 4500), TOKENS, 1),
    ((128, 1, 8, 4, 1, 500), TOKENS8, 1), ((128, 1, 8, 4, 1, 200), TOKENS, 1), ((128, 32, 8, 4, 1, 2000), TOKENS8, 1), ((128, 32, 8, 4, 1, 3000), TOKENS8, 1),
    ((128, 1, 8, 4, 1, 8000), TOKENS, 32), ((128, 16, 8, 4, 1, 30000), TOKENS, 14), ((128, 4, 8, 4, 1, 200000), TOKENS, 61), ((128, 64, 8, 4, 1, 8000), TOKENS, 3)])
def test_how_attention_is_cut(cut, sizes, kernel, parts):
    assert (cut(*sizes)[0], cut(*sizes)[2]) == (kernel, parts)


def test_every_cut_holds_all_rows_and_tokens(cut):
    rng = random.Random(1)
    for _ in range(20000):
        cols, n, heads, group = rng.choice((64, 128, 192, 256)), log(rng, 4000), log(rng, 64), log(rng, 64)
        fresh, length = log(rng, 20000), log(rng, 2 ** 31 - 512)
        kernel, groups, parts, chunk = cut(cols, n, heads, group, fresh, length)
        assert 1 <= groups <= 4096 and parts >= 1 and chunk % 256 == 0 and chunk * parts >= length > chunk * (parts - 1)
        assert parts == 1 or kernel == TOKENS
        assert kernel != TOKENS8 or cols <= 128


def test_no_estimate_makes_a_launch_too_large(cut):
    rng = random.Random(3)
    for _ in range(20000):
        cols, n, heads = rng.choice((64, 128, 192, 256)), log(rng, 65535), log(rng, 65535)
        if n * heads > 0xffffff:
            continue
        kernel, groups, parts, chunk = cut(cols, n, heads, log(rng, 128), log(rng, 2 ** 31 - 1), log(rng, 2 ** 31 - 512))
        assert groups >= 1 and n * heads * groups * parts <= 0xffffff


def log(rng, most):
    return max(1, min(most, int(most ** rng.random())))


def test_a_workspace_serves_all_smaller_calls(b, cut):
    """What the header says of abft_kv_attention_workspace_bytes, against the cut of calls of all smaller sizes."""
    rng = random.Random(2)

    def size(dim, n, heads, group, fresh, length):
        c = b.abft_kv_cache_t(None, None, None, None, 5, heads, dim, 64)
        return b.lib.abft_kv_attention_workspace_bytes(ctypes.byref(c), n, heads * group, fresh, length)
    # a layer of 16 requests of prompts up to 1100: its steps of single tokens want four parts
    assert size(128, 16, 8, 4, 1102, 1102) >= size(128, 16, 8, 4, 1, 1102) >= 4 * 16 * 32 * 130 * 4
    cut_ones = 0
    for _ in range(300):
        cols, n, heads, group = rng.choice((64, 128, 256)), log(rng, 300), rng.choice((1, 2, 5, 8, 32)), rng.choice((1, 3, 4, 8, 20))
        fresh, length = log(rng, 3000), log(rng, 300000)
        most = size(cols, n, heads, group, fresh, length)
        for _ in range(60):
            small = rng.choice((n, log(rng, n))), rng.choice((fresh, log(rng, fresh))), rng.choice((length, log(rng, length)))
            kernel, groups, parts, chunk = cut(cols, small[0], heads, group, small[1], small[2])
            assert parts == 1 or parts * small[0] * small[1] * heads * group * (cols + 2) * 4 <= most, (cols, n, heads, group, fresh, length, small)
            cut_ones += parts > 1
    assert cut_ones > 1000


def test_a_plan_in_place_is_refused(b):
    """Lengths and free blocks that overlap anything that the plan writes."""
    at = {name: 0x100000 * (i + 1) for i, name in enumerate(("ctx", "new", "table", "free", "seq", "cu", "slots", "flags", "taken"))}

    def call(**kw):
        p = {k: ctypes.c_void_p(v) for k, v in (at | kw).items()}
        return b.lib.abft_kv_plan(p["ctx"], p["new"], 4, 16, p["table"], 8, 6, p["free"], 5, p["seq"], p["cu"], p["slots"], 9, p["flags"], p["taken"], None)
    inputs, outputs = {"ctx": 16, "new": 16, "free": 20}, {"seq": 16, "cu": 20, "slots": 72, "flags": 16, "taken": 4, "table": 4 * (3 * 8 + 6)}
    for i, n in inputs.items():
        for out, m in outputs.items():
            for where in (at[i], at[i] + n - 4, at[i] - m + 4):
                assert call(**{out: where}) == b.ABFT_EINVAL and b"overlap" in b.lib.abft_last_error(), (i, out)


def test_attention_refuses_a_scale_that_overflows_in_base_two(b):
    at = ctypes.c_void_p(0x1000)
    c = b.abft_kv_cache_t(0x1000, 0x1000, 0x1000, 0x1000, 4, 2, 64, 16)
    for scale in (2.4e38, -3.4e38):
        assert b.lib.abft_kv_attention(ctypes.byref(c), at, 256, 64, 2, 3, 4, at, 8, 8, at, at, 3, 1, 100, scale, at, 256, 64, None, None, None, 0, None) == b.ABFT_EINVAL
        assert b"scale" in b.lib.abft_last_error()


# ------------------------------------------------------------------------------------- how 4-bit products are cut (csrc/w4_shape.h)
@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    """(rows, tiles of the weight, chunks of K) -> (tiles of a workgroup, its wavefronts)"""
    lib = str(tmp_path_factory.mktemp("shape") / "shape.so")
    src = ('#include "w4_shape.h"\nextern "C" void shape(int M, long long tiles, int chunks, int* out) {\n'
           '    const abft::W4Shape s = abft::w4_shape(M, tiles, chunks);\n    out[0] = s.tiles; out[1] = s.waves;\n}\n')
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", "-x", "c++", "-", "-o", lib],
                   input=src, text=True, check=True)
    so = ctypes.CDLL(lib)

    def call(M, N, K):
        out = (ctypes.c_int * 2)()
        so.shape(M, ctypes.c_longlong(-(-N // 16)), -(-K // 128), out)
        return tuple(out)
    return call


# the sizes that the rule's comment has figures of, and those on either side of where it changes
@pytest.mark.parametrize("sizes,want", [
    ((1, 4096, 4096), (1, 8)), ((16, 4096, 4096), (1, 8)), ((16, 8192, 8192), (2, 8)), ((16, 16384, 4096), (4, 8)), ((32, 16384, 4096), (4, 8)),
    ((1, 16384, 4096), (2, 8)), ((1, 4096, 16384), (1, 16)), ((4, 16384, 100), (2, 8)), ((5, 16384, 100), (4, 8)), ((1, 4096, 8064), (1, 8)),
    ((1, 4096, 8065), (1, 16)), ((1, 4097, 16384), (2, 8)), ((33, 2048, 100), (1, 8)), ((33, 2049, 100), (2, 8)), ((33, 4097, 100), (4, 8))])
def test_how_products_are_cut(shape, sizes, want):
    assert shape(*sizes) == want
