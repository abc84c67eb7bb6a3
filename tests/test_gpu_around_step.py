"""The operators around a decoding step on the GPU against step_oracle: rotated queries, codes, scales, ranks and indices equal, the rest within
the error that the oracle derives for each element."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle, step_oracle as o

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def b():
    from paper_2103_00130_amd import binding
    assert torch.cuda.is_available()
    return binding


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    return t if dtype is None else t.to(dtype)


def values(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TYPES[dtype]).cuda()


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def within(got, want, tol, what):
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        off = ~same & ~(np.abs(got - want) <= tol)
    assert not off.any(), f"{what}: {off.sum()} of {got.size} beyond the bound, first {np.argwhere(off)[0]}: {got[off][0]!r} for {want[off][0]!r} +- {np.broadcast_to(tol, got.shape)[off][0]:.3g}"


# ------------------------------------------------------------------------------------------------------------------ rotation
def rotary_case(b, rng, dtype, heads, q_heads, dim, rot, block, neighbours, fused, tokens, in_place=False, spoil=False):
    """Runs of several requests; the result against the oracle's."""
    slots, pos, blk = [], [], 0
    order = rng.permutation(tokens + 3)
    while len(slots) < tokens:
        first = int(rng.integers(0, block)) if rng.integers(0, 2) else 0
        n = min(tokens - len(slots), int(rng.integers(1, block - first + 1)) if rng.integers(0, 3) else 1)
        slots += [int(order[blk]) * block + first + i for i in range(n)]
        p0 = int(rng.integers(0, 200))
        pos += [p0 + i for i in range(n)]
        blk += 1
    slots, pos = np.array(slots, np.int64), np.array(pos, np.int32)
    n_blocks = tokens + 3
    if spoil:
        slots[rng.integers(0, tokens)] = -1
        slots[rng.integers(0, tokens)] = n_blocks * block
        pos[rng.integers(0, tokens)] = -1
        pos[rng.integers(0, tokens)] = 2 ** 31 - 1
        pos[rng.integers(0, tokens)] = 340
    c = b.KvCache(n_blocks, heads, dim, block)
    k, v = (rng.integers(-127, 128, (n_blocks, heads, block, dim)).astype(np.int8) for _ in range(2))
    ks, vs = ((rng.random((n_blocks, heads)) * 0.02).astype(np.float32) for _ in range(2))
    c.load_codes(dev(k), dev(v), dev(ks), dev(vs))
    table = b.rotary_table(340, rot, 1000.0)
    widths = (q_heads * dim, heads * dim, heads * dim)
    x = values(rng, (tokens, sum(widths) + 3 * (not fused)), dtype)
    q, kx, vx = (part.unflatten(1, (n, dim)) for part, n in zip(x[:, :sum(widths)].split(widths, 1), (q_heads, heads, heads)))
    if not fused:
        q, kx, vx = q.contiguous(), kx.transpose(0, 1).contiguous().transpose(0, 1), vx.contiguous()
    qr = q if in_place else torch.full((q_heads, tokens, dim), 5.0, dtype=TYPES[dtype], device="cuda").transpose(0, 1)
    q_before, tab = q.float().cpu().numpy(), table.cpu().numpy()
    good = (pos >= 0) & (pos < 340)
    want_q = torch.from_numpy(o.rotate(q_before, tab, pos, neighbours)).to(TYPES[dtype])
    turned = o.rotate(kx.float().cpu().numpy(), tab, pos, neighbours)
    used = np.where(good, slots, -1)
    decode_oracle.append(k, ks, turned, used)
    decode_oracle.append(v, vs, vx.float().cpu().numpy(), used)
    b.abft_kv_append_rotary(c, q, kx, vx, dev(slots), dev(pos), table, QR=None if in_place else qr, neighbours=neighbours)
    got = qr.cpu()
    assert torch.equal(got[good], want_q[good]), "queries"
    assert torch.equal(got[~good], q.cpu()[~good] if in_place else torch.full_like(got[~good], 5.0)), "queries of tokens that are left out"
    assert np.array_equal(c.k_scale.cpu().numpy(), ks) and np.array_equal(c.v_scale.cpu().numpy(), vs)
    known = np.ones((n_blocks, block), bool)      # what lies behind a run is nobody's
    last = {}
    for s in used[(used >= 0) & (used < n_blocks * block)]:
        last[int(s) // block] = int(s) % block + 1
    for i, end in last.items():
        known[i, end:] = False
    for name, g, w in zip("kv", c.codes(), (k, v)):
        assert np.array_equal(g.cpu().numpy().transpose(0, 2, 1, 3)[known], w.transpose(0, 2, 1, 3)[known]), name


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("heads,q_heads,dim,rot,block,neighbours,fused,tokens", [
    (1, 1, 2, 2, 16, False, False, 1), (2, 8, 64, 64, 16, False, True, 5), (2, 2, 64, 64, 16, True, False, 40), (3, 6, 128, 128, 64, False, True, 130),
    (5, 15, 80, 32, 16, True, True, 100), (2, 4, 33, 32, 32, False, False, 70), (1, 7, 96, 24, 64, False, True, 90), (1, 5, 96, 24, 64, True, True, 90),
    (4, 4, 48, 6, 128, False, False, 200), (2, 6, 256, 256, 128, True, False, 150), (8, 8, 128, 64, 32, False, True, 64), (3, 3, 40, 40, 16, False, False, 33),
    (3, 6, 40, 20, 16, True, False, 60), (2, 4, 256, 200, 128, False, True, 140), (2, 4, 32, 12, 32, False, False, 80), (1, 3, 8, 6, 64, True, True, 70)])
def test_rotary_append(b, dtype, heads, q_heads, dim, rot, block, neighbours, fused, tokens):
    for in_place in (False, True):
        rng = np.random.default_rng(tokens + dim + rot)
        rotary_case(b, rng, dtype, heads, q_heads, dim, rot, block, neighbours, fused, tokens, in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("neighbours", [False, True])
def test_rotary_tokens_that_are_left_out(b, neighbours, in_place):
    # (block 16 with runs of a token each where one in the middle is left out would have two runs in a block: single tokens)
    rng = np.random.default_rng(7)
    heads, q_heads, dim, block, n = 2, 6, 64, 16, 40
    c = b.KvCache(n, heads, dim, block)
    slots = rng.permutation(n).astype(np.int64) * block
    pos = rng.integers(0, 50, n).astype(np.int32)
    slots[[3, 11]], pos[[5, 6, 20]] = (-1, n * block), (-1, 50, 2 ** 31 - 1)
    table = b.rotary_table(50, dim)
    q, kx, vx = values(rng, (n, q_heads, dim), "bf16"), values(rng, (n, heads, dim), "bf16"), values(rng, (n, heads, dim), "bf16")
    kept = q.clone()
    qr = q if in_place else torch.full_like(q, 5.0)
    b.abft_kv_append_rotary(c, q, kx, vx, dev(slots), dev(pos), table, QR=qr, neighbours=neighbours)
    want = torch.from_numpy(o.rotate(kept.float().cpu().numpy(), table.cpu().numpy(), pos, neighbours)).to(torch.bfloat16)
    out = np.isin(np.arange(n), [5, 6, 20])
    assert torch.equal(qr.cpu()[~out], want[~out]) and torch.equal(qr.cpu()[out], (kept if in_place else torch.full_like(q, 5.0)).cpu()[out])
    written = np.zeros(n, bool)
    written[[s // block for t, s in enumerate(slots) if 0 <= s < n * block and not out[t]]] = True
    assert np.array_equal((c.k_scale > 0).all(1).cpu().numpy(), written) and np.array_equal((c.v_scale > 0).all(1).cpu().numpy(), written)
    assert not c.k_codes[dev(~written)].any() and not c.v_codes[dev(~written)].any()


def test_rotary_without_queries_and_with_infinities(b):
    rng = np.random.default_rng(8)
    heads, dim, block, n = 2, 32, 16, 10
    c = b.KvCache(2, heads, dim, block)
    k, v = (np.zeros((2, heads, block, dim), np.int8) for _ in range(2))
    ks, vs = (np.zeros((2, heads), np.float32) for _ in range(2))
    kx, vx = values(rng, (n, heads, dim), "f32"), values(rng, (n, heads, dim), "f32")
    kx[3, 0, 5], kx[4, 1, 20], vx[2, 0, 1] = float("inf"), float("nan"), float("-inf")
    slots, pos = np.arange(n, dtype=np.int64), np.arange(n, dtype=np.int32)
    table = b.rotary_table(n, dim)
    b.abft_kv_append_rotary(c, None, kx, vx, dev(slots), dev(pos), table)
    decode_oracle.append(k, ks, o.rotate(kx.cpu().numpy(), table.cpu().numpy(), pos, False), slots)
    decode_oracle.append(v, vs, vx.cpu().numpy(), slots)
    for g, w, gs, ws in zip(c.codes(), (k, v), (c.k_scale, c.v_scale), (ks, vs)):
        assert np.array_equal(g.cpu().numpy()[0, :, :n], w[0, :, :n]) and np.array_equal(gs.cpu().numpy(), ws)
    b.abft_kv_append_rotary(c, None, kx[:0], vx[:0], dev(slots[:0]), dev(pos[:0]), table)      # no tokens
    b.abft_kv_append_rotary(c, None, kx, vx, dev(slots), dev(pos), table[:0])                  # no position: nothing is written
    assert np.array_equal(c.k_scale.cpu().numpy(), ks)


def test_rotary_refuses_what_does_not_fit(b):
    c = b.KvCache(2, 2, 32, 16)
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")
    q, k, v, slots, pos, table = z(3, 4, 32), z(3, 2, 32), z(3, 2, 32), z(3, dtype=torch.int64), z(3, dtype=torch.int32), z(9, 32)
    for bad in ((q[:2], k, v, slots, pos, table), (q, k[:2], v, slots, pos, table), (q, k, v[:, :1], slots, pos, table), (q, k, v, slots, pos[:2], table),
                (q, k, v, slots, pos, table[:, :30]), (q, k, v, slots, pos, table[0]), (q[..., :31], k, v, slots, pos, table)):
        with pytest.raises(ValueError):
            b.abft_kv_append_rotary(c, *bad)
    for bad in ((q.half(), k, v, slots, pos, table), (q, k.half(), v, slots, pos, table), (q, k, v, slots.int(), pos, table), (q, k, v, slots, pos.long(), table),
                (q, k, v, slots, pos, table.double()), (q, k, v, slots, pos, table.cpu()), (q.cpu(), k, v, slots, pos, table)):
        with pytest.raises(TypeError):
            b.abft_kv_append_rotary(c, *bad)
    with pytest.raises(ValueError):
        b.abft_kv_append_rotary(c, None, k, v, slots, pos, table, QR=q)
    for cols in (31, 34):
        with pytest.raises(b.AbftError):
            b.abft_kv_append_rotary(c, q, k, v, slots, pos, z(9, cols))
    with pytest.raises(b.AbftError):
        b.abft_kv_append_rotary(c, q, k, v, slots, pos, table, QR=q.as_strided(q.shape, (128, 32, 1)[:1] + (0, 1)))


# ------------------------------------------------------------------------------------------------------------------ adapters
def make_pool(b, rng, dtype, K, N, ranks, max_rank, poison=True):
    """A pool whose memory held NaN before its adapters were loaded, from rows further apart than they are long; slot -1 of `ranks`: nothing loaded."""
    pool = b.LoraPool(len(ranks), K, N, max_rank, TYPES[dtype])
    if poison:
        pool.down.fill_(float("nan"))
        pool.up.fill_(float("nan"))
    plain = []
    for a, r in enumerate(ranks):
        if r < 0:
            plain.append(None)
            continue
        A, B = values(rng, (max(r, 1), K + 3), dtype)[:r, 1:K + 1], values(rng, (N, r + 2), dtype)[:, 2:]
        scale = float(rng.uniform(0.2, 2))
        pool.load(a, A if r else None, B if r else None, scale)
        plain.append((f64(A), f64(B), scale))
    return pool, plain


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,K,N,ranks,max_rank", [
    (1, 1, 1, [1], 1), (1, 640, 200, [16], 16), (2, 31, 3, [5, 0], 7), (15, 32, 64, [16, 3, 8], 16), (16, 129, 17, [17, 1], 17), (17, 5, 65, [33, -1, 128], 128),
    (40, 1000, 130, [8, 16, 2, 4, 1, 16, 16, 5, 3, 9, 16, 7, 7, 7, 7, 7, 7, 7, 16, 16], 16), (300, 264, 72, [64, 20], 64), (70, 513, 33, [31, 48], 48), (5, 4097, 16, [32, 12], 32)])
def test_lora_products(b, dtype, M, K, N, ranks, max_rank):
    rng = np.random.default_rng(M + K + N)
    pool, plain = make_pool(b, rng, dtype, K, N, ranks, max_rank)
    loaded = [a for a, r in enumerate(ranks) if r >= 0]
    for turn in range(3):
        # in any order; runs of a request's rows; with rows that have none, or one that does not exist
        ids = rng.choice(loaded + [-1, len(ranks), -2 ** 31, 2 ** 31 - 1], M) if turn == 0 else np.sort(rng.choice(loaded, M)) if turn == 1 else np.full(M, rng.choice(loaded))
        ids = ids.astype(np.int32)
        # rows further apart than they are long, off any wide alignment; or neither
        off = turn % 2
        x = values(rng, (M, K + 5 * off), dtype)[:, off:K + off]
        base, y = values(rng, (M + 1, N + 3 * off), dtype), torch.full((M + 1, N + 2 * off), 7.0, dtype=TYPES[dtype], device="cuda")
        ws = b.LoraWorkspace(pool, M).tensor
        if turn == 2:      # the least that a call takes
            ws = ws[:M * (-(-max_rank // 16) * 16)]
        ws.fill_(float("nan"))
        b.abft_lora_gemv(x, pool, dev(ids), y[:M, off:N + off], base=base[:M, :N], workspace=ws)
        want, tol = o.lora(f64(x), plain, ids, f64(base[:M, :N]), dtype)
        within(f64(y[:M, off:N + off]), want, tol, f"turn {turn}")
        assert (y[M:] == 7.0).all() and (y[:, :off] == 7.0).all() and (y[:, N + off:] == 7.0).all()
        # in place: the same bits
        z = base.clone()
        b.abft_lora_gemv(x, pool, dev(ids), z[:M, :N], workspace=ws)
        assert torch.equal(z[:M, :N], y[:M, off:N + off]) and torch.equal(z[M:], base[M:]) and torch.equal(z[:, N:], base[:, N:])


def test_lora_rows_do_not_depend_on_the_rows_beside_them(b):
    rng = np.random.default_rng(5)
    pool, _ = make_pool(b, rng, "bf16", 300, 100, [16, 4, 9], 16)
    x, base = values(rng, (33, 300), "bf16"), values(rng, (33, 100), "bf16")
    ids = rng.integers(-1, 3, 33).astype(np.int32)
    ws = b.LoraWorkspace(pool, 33).tensor
    whole, again, order = base.clone(), base.clone(), rng.permutation(33)
    b.abft_lora_gemv(x, pool, dev(ids), whole, workspace=ws)
    shuffled = base[dev(order)].contiguous()
    b.abft_lora_gemv(x[dev(order)].contiguous(), pool, dev(ids[order]), shuffled, workspace=ws)
    assert torch.equal(shuffled, whole[dev(order)])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.abft_lora_gemv(x, pool, dev(ids), again, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(again, whole)
    # an infinity and a NaN stay in their rows
    bad = x.clone()
    with_one = np.flatnonzero(ids >= 0)[:2]
    bad[with_one[0], 7], bad[with_one[1], 200] = float("inf"), float("nan")
    spoiled = base.clone()
    b.abft_lora_gemv(bad, pool, dev(ids), spoiled, workspace=ws)
    rest = np.setdiff1d(np.arange(33), with_one)
    assert torch.equal(spoiled[dev(rest)], whole[dev(rest)]) and not spoiled[dev(with_one)].isfinite().any()
    b.abft_lora_gemv(x[:0], pool, dev(ids[:0]), base[:0], workspace=ws)      # no rows


def test_lora_a_slot_is_loaded_anew_and_emptied(b):
    rng = np.random.default_rng(6)
    pool, plain = make_pool(b, rng, "f32", 50, 40, [20, 3], 20)
    x, base, ids = values(rng, (4, 50), "f32"), values(rng, (4, 40), "f32"), np.array([0, 1, 0, 1], np.int32)
    ws = b.LoraWorkspace(pool, 4).tensor
    A, B = values(rng, (2, 50), "f32"), values(rng, (40, 2), "f32")
    pool.load(0, A, B, -0.5)
    plain[0] = (f64(A), f64(B), -0.5)
    for _ in range(2):
        y = torch.empty_like(base)
        b.abft_lora_gemv(x, pool, dev(ids), y, base=base, workspace=ws)
        within(f64(y), *o.lora(f64(x), plain, ids, f64(base), "f32"), "loaded anew")
        pool.load(1, None, None)
        plain[1] = None


def test_lora_refuses_what_does_not_fit(b):
    pool = b.LoraPool(2, 64, 32, 8, torch.bfloat16)
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")
    x, y, ids, ws = z(3, 64), z(3, 32), z(3, dtype=torch.int32), b.LoraWorkspace(pool, 3).tensor
    for bad in ((x[:, :63], ids, y, None), (x, ids[:2], y, None), (x, ids, y[:2], None), (x, ids, y, y[:2]), (x, ids, y[:, :31], None)):
        with pytest.raises(ValueError):
            b.abft_lora_gemv(bad[0], pool, bad[1], bad[2], base=bad[3], workspace=ws)
    for bad in ((x.half(), ids, y, None), (x, ids.long(), y, None), (x, ids, y.float(), None), (x.cpu(), ids, y, None), (x, ids, y, y.float())):
        with pytest.raises(TypeError):
            b.abft_lora_gemv(bad[0], pool, bad[1], bad[2], base=bad[3], workspace=ws)
    for small in (None, ws[:0], ws[:40]):
        with pytest.raises(b.AbftError):
            b.abft_lora_gemv(x, pool, ids, y, workspace=small)
    with pytest.raises(ValueError):
        b.abft_lora_gemv(x, pool, ids, y, workspace=ws.repeat(2)[::2])
    for A, B, error in ((z(8, 63), z(32, 8), ValueError), (z(8, 64), z(32, 7), ValueError), (z(8, 64), None, ValueError), (z(8, 64).half(), z(32, 8), TypeError),
                        (z(9, 64), z(32, 9), b.AbftError)):
        with pytest.raises(error):
            pool.load(0, A, B)
    for slot in (-1, 2):
        with pytest.raises(b.AbftError):
            pool.load(slot, z(8, 64), z(32, 8))


# --------------------------------------------------------------------------------------------------------- log probabilities
def run_logprobs(b, x, targets, scale, top, workspace=True):
    M, V = x.shape
    new = lambda dt, *s: torch.full(s, 77, dtype=dt, device="cuda")
    out = {"logprob": new(torch.float32, M), "rank": new(torch.int32, M), "entropy": new(torch.float32, M), "lse": new(torch.float32, M)}
    tops = {"top_logprob": new(torch.float32, M, top), "top_index": new(torch.int64, M, top)}
    ws = b.LogprobsWorkspace(M, V, top).tensor if workspace else None
    if ws is not None:
        ws.fill_(float("nan"))
    b.abft_logprobs(x, dev(targets), **out, **(tops if top else {}), scale=scale, workspace=ws)
    return {k: v.cpu().numpy() for k, v in {**out, **tops}.items()}


def check_logprobs(b, x, targets, scale, top, what, workspace=True):
    got, want = run_logprobs(b, x, targets, scale, top, workspace), o.logprobs(f64(x), targets, scale, top)
    assert np.array_equal(got["rank"], want["rank"]), f"{what}: ranks {got['rank']} for {want['rank']}"
    assert np.array_equal(got["top_index"], want["top_index"]), f"{what}: alternatives, rows {np.flatnonzero((got['top_index'] != want['top_index']).any(1))}"
    for name, tol in (("logprob", "logprob_tol"), ("entropy", "entropy_tol"), ("lse", "lse_tol"), ("top_logprob", "top_tol")):
        within(got[name].astype(np.float64), want[name], want[tol], f"{what}: {name}")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,V,top", [(1, 1, 1), (3, 2, 5), (2, 7, 64), (4, 63, 3), (3, 64, 64), (5, 65, 0), (70, 100, 20), (9, 1003, 8), (2, 2048, 1), (3, 4097, 64), (6, 9001, 20),
                                     (1, 33000, 20), (2, 70001, 64), (1200, 300, 2)])
def test_logprobs(b, dtype, M, V, top):
    rng = np.random.default_rng(M + V)
    for turn in range(3):
        # whole rows; rows further apart than they are long and off any alignment; with a temperature
        x = values(rng, (M, V + 5 * (turn == 1)), dtype)[:, 3 * (turn == 1):][:, :V] * (3.0 if turn else 1.0)
        if turn == 1:
            x = torch.nn.functional.pad(x, (3, 2))[:, 3:V + 3]
        targets = rng.integers(0, V, M).astype(np.int64)
        targets[rng.random(M) < 0.2] = rng.choice([-1, V, 2 ** 40, -2 ** 62])
        check_logprobs(b, x, targets, (1.0, 1.0, 1.6)[turn], top, f"turn {turn}", workspace=turn != 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 5000, 20000])
def test_logprobs_of_masks_ties_and_orders(b, dtype, V):
    rng = np.random.default_rng(V)
    inf, lowest = float("inf"), torch.finfo(TYPES[dtype]).min
    x = torch.from_numpy(rng.standard_normal((16, V)).astype(np.float32) * 3).to(TYPES[dtype])
    some = torch.from_numpy(rng.permutation(V)[:5].copy())
    x[0] = -inf                                   # nothing is left
    x[1] = -inf
    x[1, some] = 1.0                              # a few, all the same
    x[2] = lowest                                 # the type's lowest value, which is a number
    x[3] = lowest
    x[3, some] = 2.0
    x[4] = -inf
    x[4, some[:2]] = lowest
    x[5] = 0.0                                    # all the same, with zeros of either sign
    x[5, ::3] = -0.0
    x[6] = torch.arange(V).to(x.dtype) / V * 8    # rising, with ties; falling
    x[7] = -torch.arange(V).to(x.dtype) / V * 8
    x[8] = x[8].round()                           # whole numbers: many ties
    x[9, some[0]] = float("nan")
    x[10, some[0]] = inf
    x[11] = float("nan")
    x[12] = -inf
    x[12, V - 1] = -3.0                           # one token
    x[13] = torch.finfo(TYPES[dtype]).max
    x[14, some] = torch.finfo(TYPES[dtype]).max   # far above the rest
    x[15] *= 1e-30
    x = x.cuda()
    for target in (0, V // 2, V - 1, int(some[0]), int(some[4]), -1):
        for top in (20, 64, 1):
            check_logprobs(b, x, np.full(16, target, np.int64), 1.0, top, f"target {target}, {top} alternatives")
    check_logprobs(b, x[:, 1:V - 1], np.full(16, V // 3, np.int64), 0.25, 7, "rows in rows")


def test_logprobs_parts_of_a_row_and_workspaces(b):
    """Rows cut by whatever workspace there is; results that are not asked for are not written; rows beside do not matter."""
    rng = np.random.default_rng(11)
    x = values(rng, (4, 60000), "f32")
    targets = rng.integers(0, 60000, 4).astype(np.int64)
    want = run_logprobs(b, x, targets, 1.0, 10)
    full = b.LogprobsWorkspace(4, 60000, 10).tensor
    assert full.numel() > 0 and b.LogprobsWorkspace(4, 4000, 10).tensor is None
    for n in (0, 4, 24 * 4 * 1, 24 * 4 * 2, 24 * 4 * 3 + 8, full.numel()):
        lp, ti, tl = torch.empty(4, device="cuda"), torch.empty((4, 10), dtype=torch.int64, device="cuda"), torch.empty((4, 10), device="cuda")
        guard = full.clone().fill_(3.0)
        b.abft_logprobs(x, dev(targets), logprob=lp, top_logprob=tl, top_index=ti, workspace=guard[:n])
        assert np.array_equal(ti.cpu().numpy(), want["top_index"]) and np.allclose(lp.cpu().numpy(), want["logprob"], atol=1e-4) and (guard[n:] == 3.0).all()
    lse = torch.empty(4, device="cuda")
    b.abft_logprobs(x, lse=lse)
    assert np.allclose(lse.cpu().numpy(), want["lse"], atol=1e-5)
    b.abft_logprobs(x[:0], lse=lse[:0])      # no rows
    # the same bits on another stream
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    one = torch.empty(4, device="cuda")
    b.abft_logprobs(x, dev(targets), logprob=one, workspace=full, stream=s)
    s.synchronize()
    two = torch.empty(4, device="cuda")
    b.abft_logprobs(x, dev(targets), logprob=two, workspace=full)
    assert torch.equal(one, two)


def test_logprobs_refuses_what_does_not_fit(b):
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")
    x, f, i, t = z(3, 50), z(3), z(3, dtype=torch.int32), z(3, dtype=torch.int64)
    for bad in (dict(targets=t[:2], logprob=f), dict(targets=t, logprob=f[:2]), dict(targets=t, rank=i[:2]), dict(entropy=f[:2]), dict(lse=z(6)[::2]), dict(top_logprob=z(3, 4)),
                dict(top_logprob=z(3, 4), top_index=z(3, 5, dtype=torch.int64)), dict(top_logprob=z(2, 4), top_index=z(2, 4, dtype=torch.int64))):
        with pytest.raises(ValueError):
            b.abft_logprobs(x, **bad)
    for bad in (dict(targets=i, logprob=f), dict(targets=t, logprob=f.double()), dict(targets=t, rank=t), dict(entropy=f.cpu()), dict(top_logprob=z(3, 4), top_index=z(3, 4, dtype=torch.int32))):
        with pytest.raises(TypeError):
            b.abft_logprobs(x, **bad)
    for bad in (dict(logprob=f), dict(lse=f, scale=0.0), dict(lse=f, scale=-1.0), dict(lse=f, scale=float("inf")), dict(top_logprob=z(3, 65), top_index=z(3, 65, dtype=torch.int64))):
        with pytest.raises(b.AbftError):
            b.abft_logprobs(x, **bad)
    with pytest.raises(TypeError):
        b.abft_logprobs(x.int(), lse=f)
    with pytest.raises(ValueError):
        b.abft_logprobs(x.t(), lse=f)
