"""The decoding-step operators without a GPU: the oracle against values worked out by hand or another way, and what the library
refuses on the host."""
import ctypes

import numpy as np
import pytest

from oracle import decode_oracle as o


@pytest.fixture(scope="module")
def b():
    from paper_2103_00130_amd import binding
    return binding


def test_oracle_weight_product():
    # two rows of three codes: 1 2 3 / 15 0 8, one group; the high half of the last byte is of no column
    W = np.array([[0x21, 0xF3], [0x0F, 0x78]], dtype=np.uint8)
    assert o.unpack_codes(W, 3).tolist() == [[1, 2, 3], [15, 0, 8]]
    X = np.array([[1.0, 10.0, 100.0]])
    scale, bias = np.array([[2.0], [0.5]]), np.array([[-1.0], [3.0]])
    Y, tol = o.w4_product(X, W, scale, bias, 32, "f32")
    assert Y.tolist() == [[2 * 321 - 111, 0.5 * (15 + 800) + 3 * 111]] and (tol > 0).all()
    Y, _ = o.w4_product(X, W, scale, None, 32, "f32")
    assert Y.tolist() == [[2 * (321 - 888), 0.5 * (815 - 888)]]


def test_oracle_plan():
    table = np.full((4, 3), -1)
    table[0, 0] = 9
    seq, cu, slots, flags, taken = o.plan([3, 0, 0, 5], [2, 0, 9, 1], 4, table, [20, 21, 22, 23], 12)
    # request 0 gets block 20, request 2 three blocks, request 3 finds room in the blocks it holds (two: none was written here)
    assert taken == 4 and flags.tolist() == [0, 0, 0, 0] and cu.tolist() == [0, 2, 2, 11, 12] and seq.tolist() == [5, 0, 9, 6]
    assert table.tolist() == [[9, 20, -1], [-1, -1, -1], [21, 22, 23], [-1, -1, -1]]
    assert slots.tolist() == [39, 80, 84, 85, 86, 87, 88, 89, 90, 91, 92, -3]
    table = np.full((3, 2), -1)
    seq, cu, slots, flags, taken = o.plan([0, -2, 0], [4, 12, 8], 4, table, [7, 8], 30)
    assert flags.tolist() == [0, 2 | 8, 1] and taken == 1 and seq.tolist() == [4, 0, 0]
    assert slots.tolist() == [28, 29, 30, 31] + [-1] * 26


def test_oracle_append_and_read():
    codes, scale = np.zeros((2, 1, 16, 2), np.int8), np.zeros((2, 1), np.float32)
    o.append(codes, scale, np.array([[[127.0, -63.5]], [[1.0, 0.0]]], np.float32), [16, 17])
    assert scale.tolist() == [[0.0], [1.0]] and codes[1, 0, :2].tolist() == [[127, -64], [1, 0]]
    # a larger value in the same block: the scale doubles, the codes before are halved (ties to even)
    o.append(codes, scale, np.array([[[254.0, np.nan]]], np.float32), [18])
    assert scale[1, 0] == 2 and codes[1, 0, :3].tolist() == [[64, -32], [0, 0], [127, 0]]
    assert o.read(codes, scale, [18, -1, 16, 99])[:, 0].tolist() == [[254, 0], [0, 0], [128, -64], [0, 0]]
    # offset 0 begins the block anew
    o.append(codes, scale, np.array([[[0.0, 0.0]]], np.float32), [16])
    assert scale[1, 0] == 0 and codes[1, 0, 0].tolist() == [0, 0]


def test_oracle_attention_two_ways():
    rng = np.random.default_rng(3)
    kc, vc = (rng.integers(-127, 128, (5, 2, 16, 8)).astype(np.int8) for _ in range(2))
    ks, vs = (rng.uniform(0.001, 0.02, (5, 2)).astype(np.float32) for _ in range(2))
    table, q = np.array([[3, 1], [0, 4]]), rng.standard_normal((4, 4, 8))
    O, tol, lse, _ = o.attention(q, kc, vc, ks, vs, table, [20, 0], [0, 3, 4], 0.3, "f32")
    k = np.concatenate([kc[3].astype(float) * ks[3][:, None, None], kc[1] * ks[1].astype(float)[:, None, None]], 1)[:, :20]
    v = np.concatenate([vc[3].astype(float) * vs[3][:, None, None], vc[1] * vs[1].astype(float)[:, None, None]], 1)[:, :20]
    for t in range(3):
        for i in range(4):
            z = 0.3 * (k[i // 2, :18 + t] @ q[t, i])
            w = np.exp(z) / np.exp(z).sum()
            assert np.allclose(O[t, i], w @ v[i // 2, :18 + t], rtol=1e-12) and np.isclose(lse[t, i], np.log(np.exp(z).sum()))
    assert not O[3].any() and np.all(lse[3] == -np.inf)
    assert (tol[:3] > 0).all() and tol.max() < 1e-3


def test_weight_refusals(b):
    L, d, out = b.lib, ctypes.c_void_p(0x1000), ctypes.c_void_p()
    ok = (d, 64, d, None, 1, b.ABFT_TYPE_BF16, 32, 128, 128, None, ctypes.byref(out))

    def pack(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[("W", "ldw", "scale", "bias", "lds", "type", "N", "K", "group").index(k)] = v
        return L.abft_w4_pack(*a)
    for bad in ({"W": None}, {"scale": None}, {"N": 0}, {"K": 0}, {"type": 7}, {"ldw": 63}, {"lds": 0}):
        assert pack(**bad) == b.ABFT_EINVAL, bad
    assert pack(group=48) == b.ABFT_EUNSUPPORTED and b"group=48" in L.abft_last_error()
    assert L.abft_w4_dims(None, None, None, None, None) == b.ABFT_EINVAL
    assert L.abft_w4_gemv(d, 64, 0, 1, None, d, 64, None) == b.ABFT_EINVAL
    L.abft_w4_destroy(None)


def test_plan_refusals(b):
    L, d = b.lib, ctypes.c_void_p(0x1000)
    names = ("ctx", "new", "n_req", "block", "table", "ldt", "width", "free", "n_free", "seq", "cu", "slots", "n_slots", "flags", "taken", "stream")
    ok = (d, d, 4, 16, d, 8, 8, d, 5, d, d, d, 9, d, d, None)

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[names.index(k)] = v
        return L.abft_kv_plan(*a)
    for bad in ({"ctx": None}, {"new": None}, {"n_req": -1}, {"block": 0}, {"table": None}, {"ldt": 7}, {"width": -1}, {"free": None}, {"n_free": -1},
                {"seq": None}, {"cu": None}, {"slots": None}, {"n_slots": -1}, {"flags": None}, {"taken": None}):
        assert call(**bad) == b.ABFT_EINVAL, bad
    assert call(n_req=16385) == b.ABFT_EUNSUPPORTED
    assert call(n_slots=2 ** 31 - 1) == b.ABFT_EUNSUPPORTED


def cache(b, **kw):
    f = dict(k=0x1000, v=0x1000, ks=0x1000, vs=0x1000, n_blocks=4, heads=2, dim=64, block=16)
    f.update(kw)
    return ctypes.byref(b.abft_kv_cache_t(*f.values()))


BAD_CACHES = ({"k": None}, {"v": None}, {"ks": None}, {"vs": None}, {"k": 0x1008}, {"v": 0x1004}, {"n_blocks": 0}, {"heads": 0}, {"dim": 0}, {"dim": 257},
              {"block": 8}, {"block": 48}, {"block": 256})


def test_cache_refusals(b):
    L, d = b.lib, ctypes.c_void_p(0x1000)
    assert L.abft_kv_code_bytes(cache(b, dim=80)) == 4 * 2 * 16 * 128
    assert L.abft_kv_code_bytes(cache(b, block=24)) == 0 and L.abft_kv_code_bytes(None) == 0
    for bad in BAD_CACHES:
        assert L.abft_kv_append(cache(b, **bad), d, 128, 64, d, 128, 64, 2, d, 3, None) == b.ABFT_EINVAL, bad
        assert L.abft_kv_read(cache(b, **bad), d, 3, d, 128, 64, d, 128, 64, 2, None) == b.ABFT_EINVAL, bad
    for call in (L.abft_kv_append(cache(b), d, 128, 64, d, 128, 64, 3, d, 3, None), L.abft_kv_append(cache(b), None, 128, 64, d, 128, 64, 2, d, 3, None),
                 L.abft_kv_append(cache(b), d, 128, 64, None, 128, 64, 2, d, 3, None), L.abft_kv_append(cache(b), d, 128, 64, d, 128, 64, 2, None, 3, None),
                 L.abft_kv_append(cache(b), d, 128, 64, d, 128, 64, 2, d, -1, None),
                 L.abft_kv_append(cache(b), ctypes.c_void_p(0x1001), 128, 64, d, 128, 64, 2, d, 3, None),
                 L.abft_kv_read(cache(b), None, 3, d, 128, 64, d, 128, 64, 2, None)):
        assert call == b.ABFT_EINVAL
    assert L.abft_kv_append(cache(b), None, 0, 0, None, 0, 0, 2, None, 0, None) == b.ABFT_OK   # no tokens: nothing to do
    assert L.abft_kv_append(cache(b), d, 128, 64, d, 128, 64, 2, d, 2 ** 40, None) == b.ABFT_EUNSUPPORTED


def test_attention_refusals(b):
    L, d = b.lib, ctypes.c_void_p(0x1000)
    names = ("cache", "Q", "qt", "qh", "type", "rows", "q_heads", "table", "ldt", "width", "seq", "cu", "n_req", "max_new", "max_len", "scale", "O", "ot", "oh",
             "lse", "flags", "ws", "ws_bytes", "stream")
    ok = (cache(b), d, 256, 64, 2, 3, 4, d, 8, 8, d, d, 3, 1, 100, 0.125, d, 256, 64, None, None, None, 0, None)

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[names.index(k)] = v
        return L.abft_kv_attention(*a)
    for bad in BAD_CACHES:
        assert call(cache=cache(b, **bad)) == b.ABFT_EINVAL, bad
    for bad in ({"Q": None}, {"O": None}, {"table": None}, {"seq": None}, {"cu": None}, {"type": -1}, {"rows": -1}, {"n_req": -1}, {"width": -1}, {"ldt": 7},
                {"q_heads": 0}, {"q_heads": 3}, {"max_new": 0}, {"max_len": 0}, {"scale": float("nan")}, {"scale": float("inf")},
                {"Q": ctypes.c_void_p(0x1001)}, {"O": ctypes.c_void_p(0x1001)}, {"ws": ctypes.c_void_p(0x1008), "ws_bytes": 1 << 20}):
        assert call(**bad) == b.ABFT_EINVAL, bad
    for bad in ({"n_req": 65536}, {"width": 2 ** 28, "ldt": 2 ** 28}, {"max_len": 2 ** 31 - 1}, {"rows": 2 ** 30}):
        assert call(**bad) == b.ABFT_EUNSUPPORTED, bad
    assert call(rows=0) == b.ABFT_OK and call(n_req=0) == b.ABFT_OK
    assert L.abft_kv_attention_workspace_bytes(cache(b), 3, 3, 1, 100) == 0       # query heads that do not fit
    assert L.abft_kv_attention_workspace_bytes(cache(b), 3, 4, 1, 256) == 0       # one part
    # two tokens' worth of rows, parts of 256 tokens
    assert L.abft_kv_attention_workspace_bytes(cache(b), 1, 4, 2, 1000) == 4 * (2 * 4) * (64 + 2) * 4
