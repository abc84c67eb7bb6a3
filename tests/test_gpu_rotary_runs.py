"""Rotated appends whose runs are cut by tokens that are left out, and whose workgroups look for runs among many tokens: queries, codes and scales equal to the
oracle's in every element that is a token's."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle, step_oracle
from test_gpu_around_step import TYPES, b, dev, values  # noqa: F401 (b: the fixture)

pytestmark = pytest.mark.gpu


def rotate(x, table, pos, neighbours):
    """step_oracle.rotate, all tokens at once: a product, a product, their sum, each rounded to binary32."""
    out, half = x.copy(), table.shape[1] // 2
    good = (pos >= 0) & (pos < len(table))
    c, s = (t[:, None, :] for t in np.split(table[pos[good]], 2, 1))
    i = np.arange(half)
    one, two = (2 * i, 2 * i + 1) if neighbours else (i, half + i)
    a, z = x[good][..., one], x[good][..., two]
    turned = out[good]
    with np.errstate(invalid="ignore", over="ignore"):
        turned[..., one], turned[..., two] = a * c - z * s, z * c + a * s
    out[good] = turned
    return out


def check(b, rng, dtype, heads, q_heads, dim, block, n_blocks, slots, pos, x, table, neighbours, in_place, fused=True):  # noqa: F811
    """One call on x (tokens x [queries | keys | values]) into a cache that holds something, against the oracle; the result."""
    T = len(slots)
    c = b.KvCache(n_blocks, heads, dim, block)
    k, v = (rng.integers(-127, 128, (n_blocks, heads, block, dim)).astype(np.int8) for _ in range(2))
    ks, vs = ((rng.random((n_blocks, heads)) * 0.02).astype(np.float32) for _ in range(2))
    c.load_codes(dev(k), dev(v), dev(ks), dev(vs))
    widths = (q_heads * dim, heads * dim, heads * dim)
    q, kx, vx = (p.unflatten(1, (n, dim)) for p, n in zip(x.split(widths, 1), (q_heads, heads, heads)))
    if not fused:
        q, kx, vx = q.contiguous(), kx.contiguous(), vx.contiguous()
    qr = q if in_place else torch.full((T, q_heads, dim), 5.0, dtype=TYPES[dtype], device="cuda")
    tab = table.cpu().numpy()
    kept, keys = q.cpu().clone(), kx.float().cpu().numpy()
    good = (pos >= 0) & (pos < len(tab))
    want_q = torch.from_numpy(rotate(kept.float().numpy(), tab, pos, neighbours)).to(TYPES[dtype])
    used = np.where(good, slots, -1)
    decode_oracle.append(k, ks, rotate(keys, tab, pos, neighbours), used)
    decode_oracle.append(v, vs, vx.float().cpu().numpy(), used)
    b.abft_kv_append_rotary(c, q, kx, vx, dev(slots), dev(pos), table, QR=qr, neighbours=neighbours)
    got = qr.cpu()
    assert torch.equal(got[good], want_q[good]), "queries"
    assert torch.equal(got[~good].view(torch.uint8), (kept if in_place else torch.full_like(kept, 5.0))[~good].view(torch.uint8)), "queries of tokens that are left out"
    assert np.array_equal(c.k_scale.cpu().numpy(), ks) and np.array_equal(c.v_scale.cpu().numpy(), vs)
    # what a call leaves past a run is nobody's until something is appended there: behind the last token of a block, and where tokens behind the first were left out
    known = np.ones((n_blocks, block), bool)
    for s, kept_one in zip(slots, good):
        if 0 <= s < n_blocks * block:
            if kept_one:
                known[s // block, s % block] = True
                known[s // block, s % block + 1:] = False
    for name, g, w in zip("kv", c.codes(), (k, v)):
        assert np.array_equal(g.cpu().numpy().transpose(0, 2, 1, 3)[known], w.transpose(0, 2, 1, 3)[known]), name
    return c, qr


def test_rotation_of_all_tokens_at_once_is_the_oracle():
    rng = np.random.default_rng(1)
    x, table = rng.standard_normal((9, 3, 10)).astype(np.float32), rng.standard_normal((20, 8)).astype(np.float32)
    pos = np.array([0, 19, 20, -1, 5, 5, 2 ** 31 - 1, -2 ** 31, 7])
    for neighbours in (False, True):
        assert np.array_equal(rotate(x, table, pos, neighbours), step_oracle.rotate(x, table, pos, neighbours))


# how rows are read: pairs of columns in eights; pieces of 8 columns; elements
READS = {"pairs": (32, 32, False), "pairs_part": (32, 16, False), "neighbours": (32, 32, True), "pieces": (32, 12, False), "pieces_neighbours": (40, 12, True),
         "elements": (33, 30, False), "wide": (128, 128, False)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [16, 64, 128])
@pytest.mark.parametrize("read", READS)
def test_tokens_left_out_inside_runs(b, dtype, block, read):  # noqa: F811
    """Prompts over several blocks, some of which begin inside a block.  A token that is left out cuts its run; the tokens behind it are appended behind those
    ahead of it, to the same block, whose scale they mostly raise: every token's values are larger than those before it."""
    dim, rot, neighbours = READS[read]
    heads, q_heads = 3, 6
    rng = np.random.default_rng(block + dim + rot)
    n_blocks, slots, pos = 24, [], []
    order, blk = rng.permutation(n_blocks), 0
    for first, n in ((0, 2 * block + 5), (3, block), (0, 1), (block - 1, 2), (5, 3 * block)):
        for i in range(n):
            at = first + i
            slots.append(int(order[blk + at // block]) * block + at % block)
            pos.append(i)
        blk += (first + n + block - 1) // block
    slots, pos = np.array(slots, np.int64), np.array(pos, np.int32)
    T = len(slots)
    # the first of a run, the last, one in the middle, some next to each other, every second one of a while, all of a block
    out = rng.random(T) < 0.08
    out[[0, 4, T - 1]] = True
    out[T - 3 * block:T - 2 * block] = np.arange(block) % 2 == 1
    out[2 * block + 5 + 2:2 * block + 5 + block // 2] = True
    pos[out] = rng.choice([-1, -2 ** 31, 4 * block, 2 ** 31 - 1], int(out.sum()))
    x = values(rng, (T, (q_heads + 2 * heads) * dim), dtype)
    x *= torch.linspace(0.3, 3.0, T, device="cuda").to(x.dtype)[:, None]
    x[dev(out)] = float("nan")        # (nothing of them counts)
    x[int(np.flatnonzero(out)[1])] = 3e4
    table = b.rotary_table(4 * block, rot, 1000.0)
    for in_place in (False, True):
        check(b, rng, dtype, heads, q_heads, dim, block, n_blocks, slots, pos, x.clone(), table, neighbours, in_place)


def test_no_position_is_known(b):  # noqa: F811
    """All tokens of a call are left out, with a table and with an empty one."""
    rng = np.random.default_rng(3)
    slots, pos = np.arange(100, dtype=np.int64), np.full(100, 50, np.int32)
    x = values(rng, (100, 4 * 32), "bf16")
    table = b.rotary_table(50, 32)
    for t in (table, table[:0]):
        check(b, rng, "bf16", 1, 2, 32, 16, 8, slots, pos, x, t, False, True)


# (how rows are read, heads, query heads, block, tokens, tokens among which a workgroup looks for runs)
WINDOWS = [("pairs", 8, 8, 64, 201, 2), ("pairs_part", 7, 14, 64, 501, 4), ("neighbours", 8, 16, 32, 1003, 8), ("pairs", 8, 8, 64, 1501, 16), ("pieces", 16, 16, 32, 1801, 32),
           ("pairs", 16, 16, 64, 2501, 64), ("elements", 16, 16, 128, 2333, 64), ("pieces_neighbours", 15, 15, 64, 2501, 64), ("wide", 16, 80, 128, 2200, 64),
           ("neighbours", 16, 16, 128, 2501, 64), ("pairs", 16, 32, 16, 4200, 16), ("elements", 8, 8, 16, 1100, 4), ("pieces", 3, 3, 16, 5000, 8)]


def mixed_tokens(rng, tokens, block):
    """(slots, positions, blocks): single tokens, short runs and prompts over several blocks, from anywhere in a block; some left out by their slot or position."""
    slots, pos, blk = [], [], 0
    order = rng.permutation(2 * tokens)
    while len(slots) < tokens:
        kind = rng.integers(0, 4)
        first = int(rng.integers(0, block)) if rng.integers(0, 2) else 0
        n = min(tokens - len(slots), 1 if kind < 2 else int(rng.integers(2, 9)) if kind == 2 else int(rng.integers(block, 5 * block)))
        slots += [int(order[blk + (first + i) // block]) * block + (first + i) % block for i in range(n)]
        pos += list(range(first, first + n))
        blk += (first + n + block - 1) // block
    slots, pos = np.array(slots, np.int64), np.array(pos, np.int32)
    pos[rng.random(tokens) < 0.01] = -1
    # (a slot that is outside the cache would cut a run in two: the last tokens of their blocks, and single ones)
    last = np.flatnonzero(np.append(slots[1:] != slots[:-1] + 1, True) | (slots % block == block - 1))
    slots[last[rng.random(len(last)) < 0.05]] = rng.choice([-1, 2 * tokens * block, 2 ** 62])
    return slots, pos, 2 * tokens


@pytest.mark.parametrize("dtype,in_place,fused", [("bf16", True, True), ("f32", False, True), ("f16", False, False)])
@pytest.mark.parametrize("read,heads,q_heads,block,tokens,window", WINDOWS)
def test_runs_found_among_many_tokens(b, dtype, in_place, fused, read, heads, q_heads, block, tokens, window):  # noqa: F811
    dim, rot, neighbours = READS[read]
    rng = np.random.default_rng(tokens + block + dim)
    slots, pos, n_blocks = mixed_tokens(rng, tokens, block)
    x = values(rng, (tokens, (q_heads + 2 * heads) * dim), dtype)
    check(b, rng, dtype, heads, q_heads, dim, block, n_blocks, slots, pos, x, b.rotary_table(6 * block, rot, 1000.0), neighbours, in_place, fused)


def test_a_prompt_gives_the_same_bits_every_time(b):  # noqa: F811
    """6000 tokens of one request, whose windows hold few beginnings of runs and many tokens of others'."""
    rng = np.random.default_rng(5)
    heads, q_heads, dim, block, T = 8, 32, 128, 64, 6000
    n_blocks = -(-T // block) + 3
    order = rng.permutation(n_blocks)
    t = np.arange(T)
    slots, pos = order[t // block].astype(np.int64) * block + t % block, t.astype(np.int32)
    x, table = values(rng, (T, (q_heads + 2 * heads) * dim), "bf16"), b.rotary_table(T, dim)
    c, qr = check(b, rng, "bf16", heads, q_heads, dim, block, n_blocks, slots, pos, x, table, False, False)
    q, kx, vx = (p.unflatten(1, (n, dim)) for p, n in zip(x.split((q_heads * dim, heads * dim, heads * dim), 1), (q_heads, heads, heads)))
    for _ in range(5):
        again, turned = b.KvCache(n_blocks, heads, dim, block), torch.empty_like(qr)
        b.abft_kv_append_rotary(again, q, kx, vx, dev(slots), dev(pos), table, QR=turned)
        used = torch.unique(dev(slots) // block)
        assert torch.equal(turned, qr) and torch.equal(again.k_scale[used], c.k_scale[used]) and torch.equal(again.v_scale[used], c.v_scale[used])
        for one, two in zip(again.codes(), c.codes()):
            one, two = (a[dev(slots) // block, :, dev(slots) % block] for a in (one, two))
            assert torch.equal(one, two)
