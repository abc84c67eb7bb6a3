"""The operators around a decoding step without a GPU: the oracle against values worked out another way, how work is cut, and what the
library refuses on the host."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest
import torch

from oracle import step_oracle as o


@pytest.fixture(scope="module")
def b():
    from paper_2103_00130_amd import binding
    return binding


# -------------------------------------------------------------------------------------------------------------------- oracle
def test_oracle_rotation_turns_by_the_angle():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 10)).astype(np.float32)
    angle = rng.uniform(-3, 3, (7, 4))
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    pos = [5, 0, 9]
    for neighbours in (False, True):
        y = o.rotate(x, table, pos, neighbours)
        a, c = (x[..., 0:8:2], x[..., 1:8:2]) if neighbours else (x[..., :4], x[..., 4:8])
        for t in range(2):
            z = (a[t] + 1j * c[t]) * np.exp(1j * angle[pos[t]])
            got = y[t][:, 0:8:2] + 1j * y[t][:, 1:8:2] if neighbours else y[t][:, :4] + 1j * y[t][:, 4:8]
            assert np.allclose(got, z, atol=1e-6)
        assert np.array_equal(y[2], x[2]) and np.array_equal(y[..., 8:], x[..., 8:])


def test_oracle_adapters():
    rng = np.random.default_rng(2)
    X, base = rng.standard_normal((4, 9)), rng.standard_normal((4, 5))
    A, B = rng.standard_normal((3, 9)), rng.standard_normal((5, 3))
    Y, tol = o.lora(X, [(A, B, 0.5), None], [0, -1, 1, 7], base, "f32")
    assert np.allclose(Y[0], base[0] + 0.5 * (B @ A) @ X[0]) and np.array_equal(Y[1:], base[1:])
    assert (tol > 0).all() and tol.max() < 1e-3


def test_oracle_logprobs():
    x = np.array([[0.0, np.log(2.0), np.log(3.0), np.log(2.0)], [-np.inf, 1.0, -np.inf, -np.inf], [-np.inf] * 4, [0.0, np.nan, 1.0, 2.0], [0.0, np.inf, 1.0, 2.0]])
    r = o.logprobs(x, [3, 0, 2, 1, -1], 1.0, 3)
    p = np.array([1, 2, 3, 2]) / 8
    assert np.allclose(r["logprob"][:2], [np.log(0.25), -np.inf]) and r["logprob"][2] == -np.inf and np.isnan(r["logprob"][3]) and r["logprob"][4] == 0
    assert r["rank"].tolist() == [2, 1, 2, -1, -1]
    assert np.allclose(r["entropy"][:3], [-(p * np.log(p)).sum(), 0, 0]) and np.isnan(r["entropy"][3:]).all()
    assert np.allclose(r["lse"][:2], [np.log(8), 1]) and r["lse"][2] == -np.inf
    assert r["top_index"].tolist() == [[2, 1, 3], [1, -1, -1], [-1] * 3, [-1] * 3, [-1] * 3]
    assert np.allclose(r["top_logprob"][0], np.log([3 / 8, 2 / 8, 2 / 8])) and r["top_logprob"][1].tolist() == [0.0, -np.inf, -np.inf]


# --------------------------------------------------------------------------------------------------------- how work is cut
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2103_00130_amd", "csrc")


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("cut") / "cut.so")
    src = ('#include "logprobs_cut.h"\n#include "lora_cut.h"\nextern "C" {\n'
           'int parts(long long rows, int vocab) { return abft::logprobs_parts(rows, vocab); }\n'
           'long long most_parts(long long rows, int vocab) { return abft::logprobs_most_parts(rows, vocab); }\n'
           'void lora(long long M, int K, int* out) { const abft::LoraCut c = abft::lora_cut(M, K); out[0] = c.tiles; out[1] = c.slots; out[2] = c.splits; }\n'
           'long long sums(long long M, int K, int rank) { return abft::lora_sums(M, K, rank); }\n'
           'long long most_sums(long long M, int K, int rank) { return abft::lora_most_sums(M, K, rank); }\n}\n')
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", "-x", "c++", "-", "-o", lib],
                   input=src, text=True, check=True)
    so = ctypes.CDLL(lib)
    for f in (so.most_parts, so.sums, so.most_sums):
        f.restype = ctypes.c_longlong
    so.parts.argtypes = so.most_parts.argtypes = [ctypes.c_longlong, ctypes.c_int]
    so.sums.argtypes = so.most_sums.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    so.lora.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_void_p]
    return so


def test_a_workspace_of_logprobs_serves_every_smaller_call(cuts):
    rng = random.Random(3)
    for _ in range(300):
        rows, vocab = int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 19))
        most = cuts.most_parts(rows, vocab)
        for _ in range(30):
            r, v = rng.randint(1, rows), rng.randint(1, vocab)
            n = cuts.parts(r, v)
            assert 1 <= n <= 64 and (n == 1 or r * n <= most), (rows, vocab, r, v)
    assert cuts.parts(1, 131072) == 64 and cuts.parts(5000, 131072) == 1 and cuts.parts(1024, 131072) == 1 and cuts.parts(400, 131072) == 2 and cuts.parts(1, 3000) == 1 and cuts.parts(2 ** 31 - 1, 1) == 1


def test_a_workspace_of_adapters_serves_every_smaller_call(cuts):
    rng = random.Random(4)
    out = (ctypes.c_int * 3)()
    for _ in range(60):
        M, K, rank = int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 15)), rng.randint(1, 128)
        most = cuts.most_sums(M, K, rank)
        for m in [rng.randint(1, M) for _ in range(40)] + [M]:
            assert cuts.sums(m, K, rank) <= most, (M, K, rank, m)
            cuts.lora(m, K, out)
            assert out[0] * 16 >= m > (out[0] - 1) * 16 and 1 <= out[1] <= min(16, m) and 1 <= out[2] <= 16


# ------------------------------------------------------------------------------------------------------------------ refusals
def cache(b, **kw):
    f = dict(k=0x1000, v=0x1000, ks=0x1000, vs=0x1000, n_blocks=4, heads=2, dim=64, block=16)
    f.update(kw)
    return ctypes.byref(b.abft_kv_cache_t(*f.values()))


def test_rotary_refusals(b):
    L, d, odd = b.lib, ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)
    names = ("cache", "Q", "qt", "qh", "q_heads", "QR", "rt", "rh", "K", "kt", "kh", "V", "vt", "vh", "type", "slots", "positions", "n", "table", "n_positions",
             "rot", "pairs", "stream")
    ok = (cache(b), d, 256, 64, 4, ctypes.c_void_p(0x2000), 256, 64, d, 128, 64, d, 128, 64, 2, d, d, 3, d, 100, 64, 0, None)

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[names.index(k)] = v
        return L.abft_kv_append_rotary(*a)
    for bad in ({"k": None}, {"n_blocks": 0}, {"dim": 257}, {"block": 48}):
        assert call(cache=cache(b, **bad)) == b.ABFT_EINVAL, bad
    for bad in ({"Q": None}, {"QR": None}, {"K": None}, {"V": None}, {"slots": None}, {"positions": None}, {"table": None}, {"type": 3}, {"n": -1}, {"q_heads": -1},
                {"rot": 0}, {"rot": 1}, {"rot": 63}, {"rot": 66}, {"rot": -2}, {"pairs": 2}, {"pairs": -1}, {"n_positions": -1}, {"Q": odd}, {"QR": odd}, {"K": odd}, {"V": odd},
                {"table": ctypes.c_void_p(0x1002)}, {"QR": d, "rt": 512}, {"QR": d, "rh": 128}):
        assert call(**bad) == b.ABFT_EINVAL, bad
    for bad in ({"n": 2 ** 40}, {"n_positions": 2 ** 31 + 1}, {"q_heads": 65536}):
        assert call(**bad) == b.ABFT_EUNSUPPORTED, bad
    assert call(n=0, Q=None, QR=None, K=None, V=None, slots=None, positions=None, table=None) == b.ABFT_OK


# rows of QR that lie on each other (expanded tensors) would be turned as often as they are named
@pytest.mark.parametrize("place", [0x1000, 0x2000])
@pytest.mark.parametrize("strides", [(0, 64), (256, 0), (0, 0)])
def test_rotary_refuses_rows_on_each_other(b, place, strides):
    d = ctypes.c_void_p(0x1000)
    rc = b.lib.abft_kv_append_rotary(cache(b), d, *strides, 4, ctypes.c_void_p(place), *strides, d, 128, 64, d, 128, 64, 2, d, d, 3, d, 100, 64, 0, None)
    assert rc == b.ABFT_EINVAL and b"overlap" in b.lib.abft_last_error()


def pool(b, **kw):
    f = dict(down=0x1000, up=0x1000, scale=0x1000, rank=0x1000, adapters=3, max_rank=20, K=100, N=70, type=2)
    f.update(kw)
    return ctypes.byref(b.abft_lora_t(*f.values()))


def test_lora_refusals(b):
    L, d, odd = b.lib, ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)
    down, up = ctypes.c_size_t(), ctypes.c_size_t()
    # two sixteens of ranks; four chunks of 32 columns; two blocks of 64 columns
    assert L.abft_lora_bytes(pool(b, down=None), ctypes.byref(down), ctypes.byref(up)) == b.ABFT_OK
    assert (down.value, up.value) == (3 * 2 * 4 * 1024, 3 * 2 * 2 * 2048)
    assert L.abft_lora_bytes(pool(b, type=0), ctypes.byref(down), None) == b.ABFT_OK and down.value == 3 * 2 * 7 * 1024
    sizes = ({"adapters": 0}, {"max_rank": 0}, {"max_rank": 129}, {"K": 0}, {"N": 0}, {"type": 3}, {"K": 0x7fffffff}, {"N": 0x7fffffff})
    pools = sizes + ({"down": None}, {"up": None}, {"scale": None}, {"rank": None}, {"down": 0x1008}, {"up": 0x1004})
    for bad in sizes:
        assert L.abft_lora_bytes(pool(b, **bad), None, None) == b.ABFT_EINVAL, bad
        assert L.abft_lora_workspace_bytes(pool(b, **bad), 5) == 0
    assert L.abft_lora_workspace_bytes(pool(b), 0) == 0 and L.abft_lora_workspace_bytes(pool(b), 1) == 32 * 4
    assert L.abft_lora_bytes(None, None, None) == b.ABFT_EINVAL
    names = ("pool", "slot", "A", "lda", "B", "ldb", "rank", "scale", "stream")
    ok = (pool(b), 1, d, 100, d, 20, 20, 1.0, None)

    def load(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[names.index(k)] = v
        return L.abft_lora_load(*a)
    for bad in pools:
        assert load(pool=pool(b, **bad)) == b.ABFT_EINVAL, bad
    for bad in ({"slot": -1}, {"slot": 3}, {"A": None}, {"B": None}, {"A": odd}, {"B": odd}, {"lda": 99}, {"ldb": 19}, {"rank": 21}, {"rank": -1}, {"scale": float("nan")},
                {"scale": float("inf")}):
        assert load(**bad) == b.ABFT_EINVAL, bad
    names2 = ("X", "ldx", "M", "pool", "ids", "base", "ldb", "Y", "ldy", "ws", "ws_bytes", "stream")
    ok2 = (d, 100, 5, pool(b), d, d, 70, ctypes.c_void_p(0x2000), 70, d, 1 << 20, None)

    def call(**kw):
        a = list(ok2)
        for k, v in kw.items():
            a[names2.index(k)] = v
        return L.abft_lora_gemv(*a)
    for bad in pools:
        assert call(pool=pool(b, **bad)) == b.ABFT_EINVAL, bad
    for bad in ({"X": None}, {"ids": None}, {"base": None}, {"Y": None}, {"ws": None}, {"X": odd}, {"base": odd}, {"Y": odd}, {"ldx": 99}, {"ldb": 69}, {"ldy": 69}, {"M": -1},
                {"ws": ctypes.c_void_p(0x1008)}, {"ws_bytes": 5 * 32 * 4 - 1}, {"Y": d, "ldy": 80}):
        assert call(**bad) == b.ABFT_EINVAL, bad
    assert call(M=16 * 65535 + 1) == b.ABFT_EUNSUPPORTED
    assert call(M=0, X=None, Y=None) == b.ABFT_OK


def test_logprobs_refusals(b):
    L, d, odd = b.lib, ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)
    names = ("logits", "ldl", "type", "rows", "vocab", "scale", "targets", "logprob", "rank", "entropy", "lse", "top", "top_logprob", "top_index", "ws", "ws_bytes", "stream")
    ok = (d, 100, 2, 3, 100, 1.0, d, d, d, d, d, 5, d, d, None, 0, None)

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[names.index(k)] = v
        return L.abft_logprobs(*a)
    for bad in ({"logits": None}, {"logits": odd}, {"ldl": 99}, {"type": 3}, {"rows": -1}, {"vocab": 0}, {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")},
                {"scale": float("inf")}, {"scale": 3e38}, {"targets": None}, {"top": -1}, {"top_logprob": None}, {"top_index": None}, {"ws": ctypes.c_void_p(0x1008), "ws_bytes": 64}):
        assert call(**bad) == b.ABFT_EINVAL, bad
    for bad in ({"top": 65}, {"rows": 2 ** 31}, {"vocab": 0x7fffff01, "ldl": 2 ** 31}):
        assert call(**bad) == b.ABFT_EUNSUPPORTED, bad
    assert call(rows=0, logits=None) == b.ABFT_OK
    size = L.abft_logprobs_workspace_bytes
    assert size(0, 5, 5) == 0 and size(1, 0, 5) == 0 and size(1, 5, -1) == 0 and size(1, 5, 65) == 0
    assert size(4, 3000, 5) == 0 and size(4, 100000, 5) % (16 + 40) == 0 and size(4, 100000, 5) > 0


def test_pools_and_tables_of_the_host_are_refused(b):
    for device in ("cpu", torch.device("cpu"), "meta"):
        with pytest.raises(TypeError):
            b.LoraPool(2, 64, 64, 8, device=device)
    with pytest.raises(TypeError):
        b.LoraPool(2, 64, 64, 8, torch.int8)
    for bad in ((0, 64, 64, 8), (2, 0, 64, 8), (2, 64, 0, 8), (2, 64, 64, 0), (2, 64, 64, 129)):
        with pytest.raises(ValueError):
            b.LoraPool(*bad)
    for bad in ((10, 0), (10, 7), (-1, 8)):
        with pytest.raises(ValueError):
            b.rotary_table(*bad, device="cpu")
    t = b.rotary_table(200_001, 6, 500.0, device="cpu")
    want = [np.cos(200_000 * 500.0 ** (-i / 3)) for i in range(3)] + [np.sin(200_000 * 500.0 ** (-i / 3)) for i in range(3)]
    assert t.dtype == torch.float32 and tuple(t.shape) == (200_001, 6) and np.allclose(t[-1].double().numpy(), want, atol=1e-7)
