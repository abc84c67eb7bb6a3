"""The decoding-step operators at the ends of what they take: scores, scales, lengths and estimates far from the usual."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as o

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


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def within(got, want, tol, what):
    off = np.abs(got - want) > tol
    assert not (off | ~np.isfinite(got)).any(), f"{what}: {off.sum()} of {got.size} beyond the bound, worst {np.max(np.abs(got - want) / np.maximum(tol, 1e-300)):.3g} times"


# ---------------------------------------------------------------------------------------------------------- large scores
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("block", [16, 64])
@pytest.mark.parametrize("requests,heads,group,new", [(6, 2, 4, 1), (3, 2, 3, 20), (25, 40, 1, 17)])
def test_attention_of_large_scores(b, dtype, block, requests, heads, group, new):
    """One token's score is far above all others, by so much that the weight of any other is zero: the output is that token's value,
    whatever the size and sign of the scores.  New tokens see whole tiles and parts of one."""
    rng = np.random.default_rng(block + requests)
    dim, length = 64, 192 + new
    n = -(-length // block)
    table = rng.permutation(requests * n).reshape(requests, n).astype(np.int32)
    rows = requests * new
    cu = np.arange(requests + 1, dtype=np.int32) * new
    at = rng.integers(0, 192, (requests, heads))              # the token that stands out
    sign = rng.choice([-1.0, 1.0], (requests, heads, dim))
    v = rng.integers(-127, 128, (requests * n, heads, block, dim)).astype(np.int8)
    ks, vs = ((np.exp(rng.standard_normal((requests * n, heads)) * 0.4) * 0.03).astype(np.float32) for _ in range(2))
    # rows of Q whose elements are all of one size, so that they are whole steps of their row's largest
    amp = torch.from_numpy(rng.uniform(1, 4, (rows, heads * group, 1)).astype(np.float32)).to(TYPES[dtype]).float()
    q = (amp * torch.from_numpy(np.repeat(np.repeat(sign, group, 1), new, 0).astype(np.float32))).to(TYPES[dtype]).cuda()
    who = np.repeat(np.arange(requests), new)
    for size in (1e5, 1e6, 1e7, 1e12):
        for least, most in ((20, 127), (20, -127), (-127, -60)):
            # codes along the row's signs: of others up to `least` (or all `least`), of the one `most`; a negative scale for a negative one
            near = rng.integers(-20, 21, (requests * n, heads, block, dim)).astype(np.float64)
            k = near if least == 20 else np.full(near.shape, float(least))
            scale = size / (127 * dim * 4 * 0.03) * (-1 if most == -127 else 1)
            for r in range(requests):
                for h in range(heads):
                    if least != 20:
                        for blk in table[r]:
                            k[blk, h] *= sign[r, h]
                    k[table[r, at[r, h] // block], h, at[r, h] % block] = most * sign[r, h]
            ks_now = np.full_like(ks, 0.03) if least != 20 else ks
            k = k.astype(np.int8)
            c = b.KvCache(requests * n, heads, dim, block)
            c.load_codes(dev(k), dev(v), dev(ks_now), dev(vs))
            out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
            b.abft_kv_attention(c, q, dev(table), dev(np.full(requests, length, np.int32)), dev(cu), out, new, length, scale=scale, lse=lse,
                                workspace=b.KvWorkspace(c, requests, heads * group, new, length).tensor)
            of_head = np.arange(heads * group) // group
            blk = table[who[:, None], at[who][:, of_head] // block]
            off = at[who][:, of_head] % block
            want = v[blk, of_head[None], off].astype(np.float64) * vs[blk, of_head[None]].astype(np.float64)[:, :, None]
            # a dozen roundings of binary32 (its weight is one, a whole number of steps), and the one to the type
            within(f64(out), want, np.abs(want) * (2.0 ** -19 + o.UNIT[dtype]), f"scores of {size} ({least}, {most})")
            score = (k[blk, of_head[None], off].astype(np.float64) * f64(q)).sum(2) * ks_now[blk, of_head[None]].astype(np.float64) * scale
            within(f64(lse), score, np.abs(score) * 2.0 ** -20, f"lse of scores of {size} ({least}, {most})")


# ------------------------------------------------------------------------------------------------------ lengths as estimates
@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("f32", 20)])
@pytest.mark.parametrize("workspace", [False, True])
def test_attention_with_the_longest_estimate(b, dtype, new, workspace):
    """max_len is an estimate: the largest that is taken gives the results of any other."""
    rng = np.random.default_rng(new)
    heads, group, dim, block = 2, 4, 64, 64
    lengths = np.array([700, 30, 0, 513, 1025])
    n_blocks = 40
    k, v = (rng.integers(-127, 128, (n_blocks, heads, block, dim)).astype(np.int8) for _ in range(2))
    ks, vs = ((rng.random((n_blocks, heads)) * 0.03 + 0.01).astype(np.float32) for _ in range(2))
    c = b.KvCache(n_blocks, heads, dim, block)
    c.load_codes(dev(k), dev(v), dev(ks), dev(vs))
    table = np.concatenate([rng.permutation(n_blocks)[:17] for _ in lengths]).reshape(len(lengths), 17).astype(np.int32)
    cu = (np.arange(len(lengths) + 1) * new).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((int(cu[-1]), heads * group, dim)).astype(np.float32)).to(TYPES[dtype]).cuda()
    want, tol, _, _ = o.attention(f64(q), k, v, ks, vs, table, lengths, cu, dim ** -0.5, dtype)
    longest = 2 ** 31 - 512
    ws = b.KvWorkspace(c, len(lengths), heads * group, new, longest).tensor if workspace else None
    for max_len in (longest, longest - 1, 2 ** 31 - 1200, 2 ** 30):
        out = torch.full_like(q, 9.0)
        b.abft_kv_attention(c, q, dev(table), dev(lengths.astype(np.int32)), dev(cu), out, new, max_len, workspace=ws)
        within(f64(out), want, tol, f"max_len {max_len}")


# ------------------------------------------------------------------------------------------------------------------- plans
def test_plan_refuses_lengths_past_32_bits(b):
    """A request that would hold 2^31 tokens or more is refused, though its row of the table has blocks for them: a length has 32 bits."""
    most, block = 2 ** 31 - 1, 2 ** 20
    ctx, new = [most - 3, most, 7, most - 3, 0], [3, 5, 2, 4, most]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table = torch.full((5, 2050), -1, dtype=torch.int32, device="cuda")
    table[:, :2048] = torch.arange(2048, dtype=torch.int32, device="cuda")
    free = i32([5000, 5001, 5002])
    seq, cu, flags, taken = i32([-77] * 5), i32([-77] * 6), i32([-77] * 5), i32([-77])
    slots = torch.full((16,), -77, dtype=torch.int64, device="cuda")
    b.abft_kv_plan(i32(ctx), i32(new), block, table, free, seq, cu, slots, flags, taken)
    assert flags.tolist() == [0, b.ABFT_KV_TABLE_FULL, 0, b.ABFT_KV_TABLE_FULL, b.ABFT_KV_NO_ROW]
    assert seq.tolist() == [most, most, 9, most - 3, 0] and cu.tolist() == [0, 3, 8, 10, 14, 16] and taken.tolist() == [0]
    assert slots.tolist() == [most - 3, most - 2, most - 1] + [-1] * 5 + [7, 8] + [-1] * 6
    assert (table[:, 2048:] == -1).all()


# ------------------------------------------------------------------------------------------------------ scales of values
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("heads,new", [(2, 1), (40, 17)])
def test_attention_with_scales_of_values_far_apart(b, dtype, block, heads, new):
    """Blocks whose tokens have no weight hold values that are forty orders of magnitude above those of the blocks that have all of it."""
    rng = np.random.default_rng(block + heads)
    dim, length, requests = 64, 128 + new, 25 if heads == 40 else 3
    n = -(-length // block)
    table = rng.permutation(requests * n).reshape(requests, n).astype(np.int32)
    shape = (requests * n, heads)
    k, v = (rng.integers(1, 128, shape + (block, dim)).astype(np.int8) for _ in range(2))
    ks, vs = np.zeros(shape, np.float32), np.full(shape, 1e-5, np.float32)
    low = table[:, 1]                    # the second block of every request: scores far below zero, the others' are all zero
    ks[low], vs[low] = 1.0, 1e35
    q = -torch.ones((requests * new, heads, dim)).to(TYPES[dtype]).cuda()      # (scores of -64 or less, base e, times the scale)
    c = b.KvCache(requests * n, heads, dim, block)
    c.load_codes(dev(k), dev(v), dev(ks), dev(vs))
    cu = (np.arange(requests + 1) * new).astype(np.int32)
    for scale in (5.0, 100.0, 1e10):
        out = torch.empty_like(q)
        b.abft_kv_attention(c, q, dev(table), dev(np.full(requests, length, np.int32)), dev(cu), out, new, length, scale=scale)
        want, tol, _, _ = o.attention(f64(q), k, v, ks, vs, table, [length] * requests, cu, scale, dtype)
        within(f64(out), want, tol, f"scale {scale}")
        # (weights of exactly one, whole numbers of steps, and of zero: a dozen roundings, and as many as there are tiles)
        within(f64(out), want, np.abs(want) * (2.0 ** -18 + o.UNIT[dtype]) + o.TINY[dtype], f"scale {scale}, all weights alike")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block", [16, 32, 64])
def test_attention_of_values_near_the_least(b, dtype, block):
    """Values down to 2^-103 come back like any others, in blocks of any size."""
    rng = np.random.default_rng(block)
    dim, length, heads = 64, 100, 2
    n = -(-length // block)
    table = rng.permutation(n).reshape(1, n).astype(np.int32)
    k, v = (rng.integers(1, 128, (n, heads, block, dim)).astype(np.int8) for _ in range(2))
    q = torch.from_numpy(rng.standard_normal((1, heads, dim)).astype(np.float32)).to(TYPES[dtype]).cuda()
    for least in (2.0 ** -99, 2.0 ** -101, 2.0 ** -103):
        ks, vs = np.full((n, heads), 0.001, np.float32), np.full((n, heads), least, np.float32)
        c = b.KvCache(n, heads, dim, block)
        c.load_codes(dev(k), dev(v), dev(ks), dev(vs))
        out = torch.empty_like(q)
        b.abft_kv_attention(c, q, dev(table), dev(np.array([length], np.int32)), dev(np.array([0, 1], np.int32)), out, 1, length)
        want, tol, _, _ = o.attention(f64(q), k, v, ks, vs, table, [length], [0, 1], dim ** -0.5, dtype)
        within(f64(out), want, tol, f"values of {least}")


def test_attention_of_no_rows_clears_the_flags(b):
    c = b.KvCache(4, 2, 64, 16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    q = torch.zeros((0, 4, 64), device="cuda")
    flags = torch.full((300,), 99, dtype=torch.int32, device="cuda")
    b.abft_kv_attention(c, q, i32(300, 4), i32(300), i32(301), q.clone(), 0, 0, req_flags=flags)
    assert not flags.any()


# ------------------------------------------------------------------------------------------------------ memory of the caller
def no_launch(b, monkeypatch, *names):
    """From here on a call of these library functions fails the test."""
    for name in names:
        monkeypatch.setattr(b.lib, name, lambda *a, name=name: pytest.fail(f"{name} was called"))


def test_attention_refuses_a_workspace_that_is_not_its_own_memory(b, monkeypatch):
    rng = np.random.default_rng(1)
    c = b.KvCache(64, 1, 64, 16)
    q = torch.zeros((1, 1, 64), device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table = torch.arange(64, dtype=torch.int32, device="cuda").reshape(1, 64)
    call = lambda ws: b.abft_kv_attention(c, q, table, i32([1000]), i32([0, 1]), torch.empty_like(q), 1, 1000, workspace=ws)
    size = b.abft_kv_attention_workspace_bytes(c, 1, 1, 1, 1000) // 4
    assert size > 0
    call(torch.empty(size, device="cuda"))
    no_launch(b, monkeypatch, "abft_kv_attention")
    with pytest.raises(TypeError):
        call(torch.empty(size))
    for ws in (torch.empty(1, device="cuda").expand(size), torch.empty(2 * size, device="cuda")[::2], torch.empty((size, 2), device="cuda").t()):
        with pytest.raises(ValueError):
            call(ws)


def test_checked_products_refuse_memory_that_is_not_lent_whole(b, monkeypatch):
    """The workspace of the checked GEMM and the scratch of its repairs, as attention's."""
    A = torch.zeros((8, 64), dtype=torch.uint8, device="cuda")
    Bp = b.abft_pack_b_checksum(torch.ones((64, 32), dtype=torch.int8, device="cuda"))
    C, flags = torch.zeros((8, 32), dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    ws = b.Workspace(8, Bp).tensor
    b.abft_gemm_u8s8s32_checked(A, Bp, C, flags, None, workspace=ws)
    torch.cuda.synchronize()
    no_launch(b, monkeypatch, "abft_gemm_u8s8s32_checked", "abft_workspace_init", "abft_recompute_flagged_rows", "abft_recompute_flagged_rows_async", "abft_locate_correct")
    n = ws.numel()
    for bad, error in ((torch.zeros(n, dtype=torch.int32), TypeError), (ws[:1].expand(n), ValueError), (torch.zeros(2 * n, dtype=torch.int32, device="cuda")[::2], ValueError)):
        for call in (lambda: b.abft_gemm_u8s8s32_checked(A, Bp, C, flags, None, workspace=bad), lambda: b.abft_workspace_init(bad),
                     lambda: b.abft_recompute_flagged_rows(A, Bp, C, flags, scratch=bad), lambda: b.abft_recompute_flagged_rows_async(A, Bp, C, flags, scratch=bad),
                     lambda: b.abft_locate_correct(A, Bp, C, flags, scratch=bad)):
            with pytest.raises(error):
                call()


def test_a_layer_whose_single_tokens_are_cut_after_its_prompts_were_not(b):
    """The workspace of a layer is made for its prompts; the steps of single tokens that follow are cut into parts and find room for them."""
    from paper_2103_00130_amd import decode_step
    rng = np.random.default_rng(21)
    heads, group, dim, block, hidden = 8, 4, 64, 32, 64
    rows = (heads * group + 2 * heads) * dim
    plain, handles = [], []
    for n, k in ((rows, hidden), (hidden, heads * group * dim)):
        W = rng.integers(0, 256, (n, k // 2), dtype=np.uint8)
        scale = torch.full((n, -(-k // 32)), (21.25 * k) ** -0.5)
        handles.append(b.abft_w4_pack(dev(W), scale.cuda(), (scale * -7.5).cuda(), K=k, group=32))
        plain.append((W, f64(scale), f64(scale * -7.5)))
    prompts = [1100, 900, 40, 700]
    layer = decode_step.DecodeLayer(*handles, heads * group, heads, dim, 4, 1200, sum(prompts), block, torch.float32)
    x = torch.from_numpy(rng.standard_normal((sum(prompts), hidden)).astype(np.float32)).cuda()
    layer.step(x, prompts)
    assert layer.workspace is not None
    parts = [t.cpu().numpy() for t in layer.cache.codes()]
    scales = [t.cpu().numpy() for t in (layer.cache.k_scale, layer.cache.v_scale)]
    for replayed in (False, True):
        if replayed:
            layer.record()
        layer.workspace.fill_(float("nan"))
        x = torch.from_numpy(rng.standard_normal((4, hidden)).astype(np.float32)).cuda()
        y = layer.replay(x) if replayed else layer.step(x, [1] * 4)
        assert not torch.isnan(layer.workspace).all(), "no parts were written"
        qkv, split = f64(layer.qkv[:4]), heads * group * dim
        slots, table = layer.slots[:4].cpu().numpy(), layer.table.cpu().numpy()
        for i in range(2):
            o.append(parts[i], scales[i], qkv[:, split + i * heads * dim:split + (i + 1) * heads * dim].reshape(4, heads, dim).astype(np.float32), slots)
        mid = f64(layer.mid[:4])
        want, tol, _, _ = o.attention(qkv[:, :split].reshape(4, heads * group, dim), *parts, *scales, table, layer.lengths, np.arange(5), dim ** -0.5, "f32")
        within(mid, want, tol, "attention")
        within(f64(y), *o.w4_product(mid.reshape(4, -1), *plain[1], 32, "f32"), "second projection")


@pytest.mark.parametrize("requests,heads,group,estimate", [(3, 2, 4, 1), (3, 2, 4, 2 ** 31 - 1), (25, 40, 1, 17), (25, 40, 1, 2 ** 31 - 1), (300, 250, 1, 2 ** 20)])
def test_attention_with_any_estimate_of_new_tokens(b, requests, heads, group, estimate):
    """max_new is an estimate: with one that is far too small rows are taken in turn, one that is far too large is no reason to refuse."""
    rng = np.random.default_rng(requests)
    dim, block, length, new = 16, 16, 90 if requests < 300 else 5, 80 if requests < 300 else 1
    n = -(-length // block)
    n_blocks = 3 * n
    k, v = (rng.integers(-127, 128, (n_blocks, heads, block, dim)).astype(np.int8) for _ in range(2))
    ks, vs = ((rng.random((n_blocks, heads)) * 0.03 + 0.01).astype(np.float32) for _ in range(2))
    c = b.KvCache(n_blocks, heads, dim, block)
    c.load_codes(dev(k), dev(v), dev(ks), dev(vs))
    some = min(requests, 3)     # (requests share blocks, and those past the third have one new token: the oracle takes its time)
    table = np.stack([np.arange(n) + n * (r % some) for r in range(requests)]).astype(np.int32)
    fresh = np.array([new if r < some else 1 for r in range(requests)])
    cu = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((int(cu[-1]), heads * group, dim)).astype(np.float32)).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    b.abft_kv_attention(c, q, dev(table), dev(np.full(requests, length, np.int32)), dev(cu), out, estimate, length,
                        workspace=b.KvWorkspace(c, requests, heads * group, estimate, length).tensor)
    last = min(requests, 6)
    rows = int(cu[last])
    want, tol, _, _ = o.attention(f64(q[:rows]), k, v, ks, vs, table[:last], [length] * last, cu[:last + 1], dim ** -0.5, "bf16")
    within(f64(out[:rows]), want, tol, f"{requests} requests, max_new {estimate}")


def test_a_step_that_is_refused_leaves_the_layer_as_it_was(b):
    from paper_2103_00130_amd import decode_step
    g = torch.Generator("cuda").manual_seed(1)
    handles = [decode_step.random_weight(n, 64, 32, torch.float32, g) for n in (192, 64)]
    layer = decode_step.DecodeLayer(*handles, 1, 1, 64, 2, 30, 20, 16, torch.float32)
    x = torch.zeros((2, 64), device="cuda")
    with pytest.raises(RuntimeError):
        layer.replay(x)
    layer.record()
    for bad, error in ((x.half(), TypeError), (x.cpu(), TypeError), (x[:, :63], ValueError), (x[:1], ValueError), (torch.zeros((64, 2), device="cuda").t(), ValueError)):
        with pytest.raises(error):
            layer.step(bad, [1, 1])
    for bad in (x[:1], x[:, :63]):
        with pytest.raises(ValueError):
            layer.replay(bad)
    assert layer.lengths == [0, 0] and layer.used == 0 and not layer.ctx.any()
    layer.step(x, [1, 1])
    assert layer.lengths == [1, 1] and layer.used == 2 and layer.ctx.tolist() == [1, 1]


# ----------------------------------------------------------------------------------------------------------- 4-bit weights
@pytest.mark.parametrize("dtype,scale_dtype", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "f16"), ("f16", "bf16")])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_products_of_wide_and_of_long_weights(b, dtype, scale_dtype, group):
    """Sizes on both sides of every change of the cut: several tiles of the weight to a workgroup, the last one with fewer; sixteen wavefronts; many rows."""
    sizes = [(1, 4100, 100), (4, 4161, 131), (5, 4100, 257), (16, 4113, 1300), (17, 4100, 129), (33, 4099, 65), (1, 8300, 33), (5, 8300, 300), (16, 8241, 129),
             (33, 2050, 130), (1, 40, 8065), (4, 17, 8200), (5, 33, 8191), (16, 16, 8320), (20, 16, 8200), (200, 50, 300), (513, 17, 260)]
    for case, (M, N, K) in enumerate(sizes):
        rng = np.random.default_rng(1000 * group + case)
        G = -(-K // group)
        W = rng.integers(0, 256, (N, (K + 1) // 2), dtype=np.uint8)
        scale = torch.from_numpy((np.exp(rng.standard_normal((N, G)) * 0.5) * 0.05).astype(np.float32)).to(TYPES[scale_dtype])
        shift = torch.from_numpy((rng.standard_normal((N, G)) * 0.5).astype(np.float32)).to(TYPES[scale_dtype]) if (case + group // 32) % 2 else None
        x = torch.from_numpy(rng.standard_normal((M, K + 1)).astype(np.float32)).to(TYPES[dtype]).cuda()[:, case % 2:][:, :K]
        y = torch.full((M, N + 1), 7.0, dtype=TYPES[dtype], device="cuda")
        Wp = b.abft_w4_pack(dev(W), scale.cuda(), None if shift is None else shift.cuda(), K=K, group=group)
        b.abft_w4_gemv(x, Wp, y[:, :N])
        want, tol = o.w4_product(f64(x), W, f64(scale), None if shift is None else f64(shift), group, dtype)
        within(f64(y[:, :N]), want, tol, f"{M}x{N}x{K} group {group}")
        assert (y[:, N:] == 7.0).all()


# ------------------------------------------------------------------------------------------- kernels and batches of attention
def held(b, rng, lengths, fresh, heads, group, dim, block, dtype):
    """(cache, its parts, table, cu_new, q) of requests whose blocks lie in no order"""
    n = [-(-int(x) // block) for x in lengths]
    n_blocks = sum(n) + 2
    k, v = (rng.integers(-127, 128, (n_blocks, heads, block, dim)).astype(np.int8) for _ in range(2))
    ks, vs = ((rng.random((n_blocks, heads)) * 0.03 + 0.01).astype(np.float32) for _ in range(2))
    c = b.KvCache(n_blocks, heads, dim, block)
    c.load_codes(dev(k), dev(v), dev(ks), dev(vs))
    ids, table, at = rng.permutation(n_blocks), np.full((len(lengths), max(n)), -1, np.int32), 0
    for r, m in enumerate(n):
        table[r, :m] = ids[at:at + m]
        at += m
    cu = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((int(cu[-1]), heads * group, dim)).astype(np.float32)).to(TYPES[dtype]).cuda()
    return c, (k, v, ks, vs), table, cu, q


@pytest.mark.parametrize("dim,block", [(64, 64), (128, 16), (90, 32)])
def test_eight_wavefronts_in_binary16(b, dim, block):
    rng = np.random.default_rng(dim)
    lengths = rng.integers(1, 1000, 13)
    lengths[3] = 1000
    c, parts, table, cu, q = held(b, rng, lengths, [1] * 13, 10, 2, dim, block, "f16")
    out = torch.empty_like(q)
    b.abft_kv_attention(c, q, dev(table), dev(lengths.astype(np.int32)), dev(cu), out, 1, 1000)
    want, tol, _, _ = o.attention(f64(q), *parts, table, lengths, cu, dim ** -0.5, "f16")
    within(f64(out), want, tol, "eight wavefronts")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,group,block", [(2, 4, 64), (40, 1, 16), (3, 7, 32)])
def test_prompts_and_single_tokens_in_one_call(b, dtype, heads, group, block):
    """One prompt, a part of one, a request that waits and single tokens of long and short requests."""
    rng = np.random.default_rng(heads)
    lengths = np.array([700, 130, 1, 0, 64, 90, 65, 333] + [40] * (18 if heads == 40 else 0))
    fresh = np.array([1, 130, 1, 0, 1, 37, 0, 1] + [1] * (len(lengths) - 8))
    c, parts, table, cu, q = held(b, rng, lengths, fresh, heads, group, 32, block, dtype)
    want, tol, want_lse, lse_tol = o.attention(f64(q), *parts, table, lengths, cu, 32 ** -0.5, dtype)
    for estimate in (130, 1):
        out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda")
        ws = b.KvWorkspace(c, len(lengths), heads * group, 130, 700).tensor
        b.abft_kv_attention(c, q, dev(table), dev(lengths.astype(np.int32)), dev(cu), out, estimate, 700, lse=lse, workspace=ws)
        within(f64(out), want, tol, f"estimate {estimate}")
        within(f64(lse), want_lse, lse_tol, f"lse, estimate {estimate}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 128])
def test_products_of_large_elements(b, dtype, group):
    """Elements just below 2^115, all of one sign, and rows with an infinity beside a weight that is positive everywhere."""
    rng = np.random.default_rng(group)
    M, N, K = 5, 40, 256
    W = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    scale = torch.full((N, K // group), 0.01)
    for bias in (None, torch.full((N, K // group), -0.075), torch.full((N, K // group), 0.5)):
        Wp = b.abft_w4_pack(dev(W), scale.cuda(), None if bias is None else bias.cuda(), K=K, group=group)
        x = torch.from_numpy((rng.uniform(1, 1.99, (M, K)) * 2.0 ** 114).astype(np.float32)).to(TYPES[dtype]).cuda()
        y = torch.empty((M, N), dtype=TYPES[dtype], device="cuda")
        b.abft_w4_gemv(x, Wp, y)
        want, tol = o.w4_product(f64(x), W, f64(scale), None if bias is None else f64(bias), group, dtype)
        within(f64(y), want, tol, "large elements")
        x = torch.ones((M, K), dtype=TYPES[dtype], device="cuda")
        x[1, 3], x[4, 255] = float("inf"), float("nan")
        b.abft_w4_gemv(x, Wp, y)
        finite = np.isfinite(f64(y)).all(1)
        assert finite.tolist() == [True, False, True, True, False] and not np.isfinite(f64(y)[[1, 4]]).any()
