"""Operators of a decoding step around its products and its attention, as cases that can be timed and compared.

Each case is one pass through one operator at one size:

* ``rotary``    queries and keys of new tokens rotated by their positions, keys and values quantized into the 8-bit cache on the way, and
                the blocks they went to read back as values (`abft_kv_append_rotary`, `abft_kv_read`),
* ``lora``      low-rank adapters of many requests at once, added to what a shared projection gave (`abft_lora_gemv`),
* ``logprobs``  log probabilities of given tokens, their ranks, the rows' entropy and the most probable tokens (`abft_logprobs`).

`listed()` names the sizes that stand for each kind of use, `draw()` gives more sizes of the same ranges, `prepare()` makes what a
program holds before the call, `run()` is the call: the plain form in torch where `own` is false, the library's where it is true.
`exact()` evaluates the definitions in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
TINY = 2.0 ** -126          # the smallest scale of a block that holds a value other than zero
MOST_ROTARY = 6000 * (32 + 2 * 8) * 128      # elements of the largest listed prompt
MOST_LORA = 4096 * (4096 + 2 * 4096)         # elements of X, base and Y of prompts about as long as the largest listed ones
MOST_LOGITS = 2048 * 32000


# ---------------------------------------------------------------------------------------------------------------- cases
def rotary(name, requests, longest, new, q_heads, heads, dim, rot, block, dtype="bf16", neighbours=False, fused=False):
    """New tokens of `requests` requests (one each, or up to `new`) behind up to `longest` that are there; `rot` columns of a head turn,
    in pairs of neighbours or of one column from either half.  fused: Q, K and V are slices of the rows of a fused projection."""
    return {"name": name, "op": "rotary", "requests": requests, "longest": longest, "new": new, "q_heads": q_heads, "heads": heads,
            "dim": dim, "rot": rot, "block": block, "dtype": dtype, "neighbours": neighbours, "fused": fused}


def lora(name, requests, new, K, N, adapters, rank, dtype="bf16", odd=False):
    """Rows of `requests` requests (one each, or up to `new`), each with one of `adapters` adapters or with none, K columns to N.  The
    ranks go up to `rank`: halves and quarters of it, or any (odd)."""
    return {"name": name, "op": "lora", "requests": requests, "new": new, "K": K, "N": N, "adapters": adapters, "rank": rank,
            "dtype": dtype, "odd": odd}


def logprobs(name, rows, vocab, top, dtype="f32", temperature=1.0, masked=False):
    """Rows of logits.  masked: in half of the rows all but some hundred tokens are ruled out, as by a grammar; in one all are."""
    return {"name": name, "op": "logprobs", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "temperature": temperature,
            "masked": masked}


def listed():
    return [
        # the new token of one request: a call where latency is everything
        rotary("rotary_step_1", 1, 777, 1, 32, 8, 128, 128, 64),
        # the new token of each request of a decoding step, sliced out of a fused projection
        rotary("rotary_step_64", 64, 4000, 1, 32, 8, 128, 128, 64, fused=True),
        # a prompt of several thousand tokens
        rotary("rotary_prompt_6000", 1, 0, 6000, 32, 8, 128, 128, 64, fused=True),
        # prompts and their continuations of uneven length; a head of 80 columns of which 32 turn, as neighbours
        rotary("rotary_mixed_40", 40, 1000, 300, 15, 5, 80, 32, 16, dtype="f16", neighbours=True),
        # one token through one adapter: latency
        lora("lora_step_1", 1, 1, 4096, 4096, 4, 16),
        # a decoding batch whose requests use many adapters, beside the fused projection of queries, keys and values
        lora("lora_step_64", 64, 1, 4096, 6144, 48, 16),
        # prompts of several requests through their adapters
        lora("lora_prompts_9", 9, 2048, 4096, 4096, 4, 32),
        # sizes without a factor in common with anything, in 32 bits
        lora("lora_odd_11", 11, 6, 1237, 5001, 5, 13, dtype="f32", odd=True),
        # the token that was sampled from one row, with its alternatives: latency
        logprobs("logprobs_1x131072", 1, 131072, 20, dtype="bf16"),
        # a decoding batch, some of it under a grammar
        logprobs("logprobs_64x50001", 64, 50001, 8, dtype="f16", temperature=0.7, masked=True),
        # a prompt's tokens scored
        logprobs("logprobs_2048x32000", 2048, 32000, 5),
        # scores alone, of a small vocabulary
        logprobs("logprobs_300x1003", 300, 1003, 0, dtype="bf16", temperature=1.3),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("rotary", "lora", "logprobs"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op == "rotary":
        heads, dim = rng.choice((1, 2, 3, 5, 8, 16)), rng.choice((32, 64, 64, 80, 96, 128, 128, 128, 192, 256))
        q_heads = heads * rng.choice((1, 2, 4, 4, 7, 8))
        rot = rng.choice((dim, dim, dim, dim // 2, dim // 4, 2 * rng.randint(1, dim // 2)))
        requests = _log_int(rng, 1, 256)
        es = 2 if dtype == "f32" else 1
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(2, MOST_ROTARY // ((q_heads + 2 * heads) * dim * requests * es)))
        longest = _log_int(rng, 1, max(1, min(8000, 400_000_000 // (requests * heads * dim * 2))))
        return rotary("drawn", requests, longest, new, q_heads, heads, dim, rot, rng.choice((16, 32, 64, 128)), dtype, rng.random() < 0.3, rng.random() < 0.5)
    if op == "lora":
        K, N = _log_int(rng, 16, 16384), _log_int(rng, 16, 16384)
        if rng.random() < 0.6:
            K, N = (K + 63) // 64 * 64, (N + 63) // 64 * 64
        rank = rng.choice((4, 8, 16, 16, 32, 64, 128, rng.randint(1, 128)))
        adapters = _log_int(rng, 1, max(1, min(64, 8_000_000 // (rank * (K + N)))))
        requests = _log_int(rng, 1, 128)
        # (neither the rows' elements nor their products beyond those of the largest listed prompts)
        most = min(MOST_LORA // (K + 2 * N), MOST_LORA * 18 // ((K + N) * rank)) // (2 if dtype == "f32" else 1)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(2, min(4096, most) // requests))
        return lora("drawn", requests, new, K, N, adapters, rank, dtype, odd=rng.random() < 0.5)
    vocab = _log_int(rng, 100, 262144)
    rows = _log_int(rng, 1, max(1, min(8192, MOST_LOGITS // vocab)))
    return logprobs("drawn", rows, vocab, rng.choice((0, 1, 5, 8, 20, 20, 64)), dtype, rng.choice((1.0, 1.0, 0.7, 1.5)), rng.random() < 0.4)


# --------------------------------------------------------------------------------------------------------------- inputs
def _ceil(a, b):
    return -(-a // b)


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)


def _sizes_seed(case):
    """What the lengths, ranks and adapters of a case are drawn from: its sizes alone."""
    return np.random.RandomState(sum(v * p for v, p in zip((v for v in case.values() if type(v) is int), (7919, 31, 7, 101, 13, 1009, 3, 17))) % (2 ** 32))


def _fresh(case, rs):
    """New tokens of each request."""
    R, new = case["requests"], case["new"]
    fresh = np.ones(R, dtype=np.int64)
    if new > 1:
        if R == 1:
            fresh[:] = new
        else:
            kind = rs.uniform(size=R)
            prompt = np.exp(rs.uniform(0, math.log(new + 1), R)).astype(np.int64)
            fresh = np.where(kind < 0.7, np.maximum(prompt, 1), np.where(kind < 0.9, 1, 0))
            fresh[rs.randint(R)] = new
    return fresh


def _lengths(case):
    rs = _sizes_seed(case)
    ctx = rs.randint(0, case["longest"] + 1, case["requests"]).astype(np.int64)
    return ctx, _fresh(case, rs)


def _adapters(case):
    """(ranks of the adapters, new tokens and adapter of each request, -1: none)"""
    rs = _sizes_seed(case)
    fresh, n, rank = _fresh(case, rs), case["adapters"], case["rank"]
    ranks = rs.randint(1, rank + 1, n) if case["odd"] else np.maximum(rank >> rs.choice((0, 0, 1, 2), n), 1)
    ranks[rs.randint(n)] = rank
    which = rs.randint(0, n, case["requests"])
    which[rs.uniform(size=case["requests"]) < 0.1] = -1
    which[np.argmax(fresh)] = np.argmax(ranks)
    return ranks.astype(np.int64), fresh, which


def _inputs(case, seed):
    """What both sides start from."""
    rs = np.random.RandomState(seed % (2 ** 32))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return {"rotary": _rotary_inputs, "lora": _lora_inputs, "logprobs": _logprobs_inputs}[case["op"]](case, rs, gen) | {"case": case}


def _rotary_inputs(case, rs, gen):
    order = rs.permutation(case["requests"])
    ctx, fresh = (x[order] for x in _lengths(case))
    total, block = ctx + fresh, case["block"]
    have = _ceil(total, block)
    n_blocks = int(have.sum()) + 7
    ids, begin = rs.permutation(n_blocks), np.concatenate([[0], np.cumsum(have)])
    slot = lambda r, p: ids[begin[r] + p // block].astype(np.int64) * block + p % block
    join = lambda parts: np.concatenate(parts) if parts else np.empty(0, dtype=np.int64)
    where = [np.arange(c, t) for c, t in zip(ctx, total)]
    held = [np.arange(c // block * block, t) if t > c else np.arange(0) for c, t in zip(ctx, total)]
    slots, back = join([slot(r, p) for r, p in enumerate(where)]), join([slot(r, p) for r, p in enumerate(held)])
    heads, q_heads, dim, dt, T = case["heads"], case["q_heads"], case["dim"], TYPES[case["dtype"]], int(fresh.sum())
    st = {"slots": torch.tensor(slots, device=DEV), "back": torch.tensor(back, device=DEV), "n_blocks": n_blocks,
          "positions": torch.tensor(join(where).astype(np.int32), device=DEV)}
    # angles of every position that there may be, in 64 bits, as cosines and sines in 32
    rot = case["rot"]
    angle = torch.arange(case["longest"] + case["new"] + 1, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    st["table"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    for name in ("k", "v"):
        codes = torch.randn((n_blocks, heads, block, dim), generator=gen, device=DEV).mul_(36).round_().clamp_(-127, 127)
        st[name], st[name + "s"] = codes.to(torch.int8), torch.exp(0.3 * _randn(gen, n_blocks, heads)) * (3.5 / 127)
    widths = (q_heads * dim, heads * dim, heads * dim)
    x = (_randn(gen, T, sum(widths)) * torch.exp(0.4 * _randn(gen, T, 1))).to(dt)
    for name, part, n in zip(("q", "kx", "vx"), x.split(widths, 1), (q_heads, heads, heads)):
        st[name] = (part if case["fused"] else part.contiguous()).unflatten(1, (n, dim))
    return st


def _lora_inputs(case, rs, gen):
    ranks, fresh, which = _adapters(case)
    order = rs.permutation(case["requests"])
    fresh, which = fresh[order], which[order]
    ids = np.repeat(which, fresh)
    M, K, N, n, R, dt = len(ids), case["K"], case["N"], case["adapters"], case["rank"], TYPES[case["dtype"]]
    live = torch.arange(R, device=DEV)[None, :] < torch.tensor(ranks, device=DEV)[:, None]     # [adapter][rank]
    return {"ids": torch.tensor(ids, dtype=torch.int32, device=DEV), "ranks": ranks.tolist(), "live": live,
            "x": (_randn(gen, M, K) * torch.exp(0.5 * _randn(gen, 1, K))).to(dt), "base": _randn(gen, M, N).to(dt),
            "down": (_randn(gen, n, R, K) / math.sqrt(K) * live[:, :, None]).to(dt), "up": (0.3 * _randn(gen, n, N, R) * live[:, None, :]).to(dt),
            "scale": [16.0 / int(r) for r in np.maximum(ranks, 8)]}


def _logprobs_inputs(case, rs, gen):
    M, V, dt = case["rows"], case["vocab"], TYPES[case["dtype"]]
    # scores of a few units, and some tokens far above the rest; from rows that are nearly sure to rows that are not
    x = _randn(gen, M, V).mul_(2.0).add_(_randn(gen, M, 1))
    some = torch.randint(0, V, (M, 40), generator=gen, device=DEV)
    x.scatter_add_(1, some, 8.0 * torch.rand((M, 40), generator=gen, device=DEV) * (1.5 * torch.rand((M, 1), generator=gen, device=DEV)))
    # targets: a likely token, any token, none
    kind = torch.rand(M, generator=gen, device=DEV)
    targets = torch.where(kind < 0.6, some[:, 0], torch.randint(0, V, (M,), generator=gen, device=DEV))
    if M > 4:
        targets[torch.rand(M, generator=gen, device=DEV) < 0.05] = -1
    if case["masked"]:
        allowed = torch.rand((M, V), generator=gen, device=DEV) < 100.0 / V
        allowed.scatter_(1, some[:, :1], True)
        allowed |= torch.rand((M, 1), generator=gen, device=DEV) < 0.5
        if M > 2:
            allowed[int(rs.randint(M))] = False
        x.masked_fill_(~allowed, -math.inf)
    return {"logits": x.to(dt), "targets": targets, "scale": 1.0 / case["temperature"]}


def prepare(case, seed):
    st = _inputs(case, seed)
    st["own"] = own
    if not own:
        return st
    from paper_2103_00130_amd import binding as b
    if case["op"] == "rotary":
        cache = b.KvCache(st.pop("n_blocks"), case["heads"], case["dim"], case["block"])
        cache.load_codes(st.pop("k"), st.pop("v"), st.pop("ks"), st.pop("vs"))
        shape = (st["back"].numel(), case["heads"], case["dim"])
        st.update(cache=cache, qr=torch.empty(st["q"].shape, dtype=st["q"].dtype, device=DEV))
        st["k_back"], st["v_back"] = (torch.empty(shape, dtype=st["kx"].dtype, device=DEV) for _ in range(2))
    elif case["op"] == "lora":
        pool = b.LoraPool(case["adapters"], case["K"], case["N"], case["rank"], TYPES[case["dtype"]])
        down, up = st.pop("down"), st.pop("up")
        for a, r in enumerate(st["ranks"]):
            pool.load(a, down[a, :r], up[a, :, :r], st["scale"][a])
        st.update(pool=pool, y=torch.empty_like(st["base"]), ws=b.LoraWorkspace(pool, st["x"].shape[0]))
    else:
        M, top = case["rows"], case["top"]
        new = lambda dt, *shape: torch.empty(shape, dtype=dt, device=DEV)
        st.update(logprob=new(torch.float32, M), rank=new(torch.int32, M), entropy=new(torch.float32, M), lse=new(torch.float32, M),
                  top_logprob=new(torch.float32, M, top), top_index=new(torch.int64, M, top), ws=b.LogprobsWorkspace(M, case["vocab"], top))
    return st


# ----------------------------------------------------------------------------------------------------------------- runs
def run(st):
    op = st["case"]["op"]
    if st["own"]:
        return _OWN[op](st)
    return _PLAIN[op](st)


def _own_rotary(st):
    from paper_2103_00130_amd import binding as b
    b.abft_kv_append_rotary(st["cache"], st["q"], st["kx"], st["vx"], st["slots"], st["positions"], st["table"], QR=st["qr"], neighbours=st["case"]["neighbours"])
    b.abft_kv_read(st["cache"], st["back"], st["k_back"], st["v_back"])
    return {"q": st["qr"], "k": st["k_back"], "v": st["v_back"], "k_scale": st["cache"].k_scale, "v_scale": st["cache"].v_scale}


def _own_lora(st):
    from paper_2103_00130_amd import binding as b
    b.abft_lora_gemv(st["x"], st["pool"], st["ids"], st["y"], base=st["base"], workspace=st["ws"].tensor)
    return st["y"]


def _own_logprobs(st):
    from paper_2103_00130_amd import binding as b
    out = {name: st[name] for name in ("logprob", "rank", "entropy", "lse", "top_logprob", "top_index")}
    b.abft_logprobs(st["logits"], st["targets"], **out, scale=st["scale"], workspace=st["ws"].tensor)
    return out


_OWN = {"rotary": _own_rotary, "lora": _own_lora, "logprobs": _own_logprobs}


def _plain_turn(x, table, positions, neighbours):
    """The first columns of x turned by their tokens' angles, in 32 bits."""
    x = x.float()
    cos, sin = table[positions.long()][:, None, :].chunk(2, 2)
    half = cos.shape[2]
    a, b = (x[..., :2 * half:2], x[..., 1:2 * half:2]) if neighbours else (x[..., :half], x[..., half:2 * half])
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([c, d], 3).flatten(2) if neighbours else torch.cat([c, d], 2)
    return torch.cat([turned, x[..., 2 * half:]], 2)


def _plain_quantize(codes, scale, x, slots, block):
    """New rows x [T][heads][dim] into codes and scale, in place."""
    blk, off = slots // block, slots % block
    touched, seg = torch.unique_consecutive(blk, return_inverse=True)
    n = touched.numel()
    start = torch.full((n,), block, device=DEV, dtype=torch.int64).scatter_reduce(0, seg, off, "amin")
    peak = torch.zeros((n, x.shape[1]), device=DEV).index_reduce_(0, seg, x.abs().amax(2), "amax")
    fresh = torch.where(peak > 0, torch.clamp(peak / 127, min=TINY), 0.0)
    old = torch.where((start > 0)[:, None], scale[touched], 0.0)
    s = torch.maximum(old, fresh)
    ratio = torch.where(s > 0, old / s, 1.0)
    held = codes[touched].float()
    before = torch.arange(block, device=DEV)[None, None, :, None] < start[:, None, None, None]
    codes[touched] = torch.where(before, torch.round(held * ratio[:, :, None, None]), held).to(torch.int8)
    inv = torch.where(s > 0, 1.0 / s, 0.0)
    codes[blk, :, off] = torch.round(x * inv[seg][:, :, None]).clamp(-127, 127).to(torch.int8)
    scale[touched] = s


def _plain_rotary(st):
    case, dt = st["case"], st["q"].dtype
    block = case["block"]
    q = _plain_turn(st["q"], st["table"], st["positions"], case["neighbours"]).to(dt)
    _plain_quantize(st["k"], st["ks"], _plain_turn(st["kx"], st["table"], st["positions"], case["neighbours"]), st["slots"], block)
    _plain_quantize(st["v"], st["vs"], st["vx"].float(), st["slots"], block)
    blk, off = st["back"] // block, st["back"] % block
    return {"q": q, "k": (st["k"][blk, :, off].float() * st["ks"][blk][:, :, None]).to(dt),
            "v": (st["v"][blk, :, off].float() * st["vs"][blk][:, :, None]).to(dt), "k_scale": st["ks"], "v_scale": st["vs"]}


def _plain_lora(st):
    # all adapters side by side: a row keeps the ranks of its own
    n, N, R = st["up"].shape
    mine = (st["ids"][:, None] == torch.arange(n, device=DEV)) * torch.tensor(st["scale"], device=DEV)        # [row][adapter]
    mid = (st["x"].float() @ st["down"].float().reshape(n * R, -1).t()).unflatten(1, (n, R)) * mine[:, :, None]
    return (st["base"].float() + mid.flatten(1) @ st["up"].float().transpose(1, 2).reshape(n * R, N)).to(st["base"].dtype)


def _plain_logprobs(st):
    x, scale, t, top = st["logits"].float(), st["scale"], st["targets"], st["case"]["top"]
    M, V = x.shape
    highest = x.amax(1, keepdim=True)
    some = highest > -math.inf
    d = (x - torch.where(some, highest, 0.0)) * scale
    e = torch.exp(d)
    total = torch.where(some, e.sum(1, keepdim=True), 1.0)
    log_total = torch.log(total)
    lse = torch.where(some, highest * scale + log_total, -math.inf)
    entropy = torch.where(some, log_total - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total, 0.0)
    inside = (t >= 0) & (t < V)
    at = torch.where(inside, t, 0)[:, None]
    index = torch.arange(V, device=DEV)
    mine = x.gather(1, at)
    rank = ((x > mine) | ((x == mine) & (index < at))).sum(1)
    # one whole number orders by value, then by the lower index
    bits = (x + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2 ** 32 + (2 ** 31 - index)
    first = key.topk(min(top, V), 1).values
    first = torch.cat([first, first.new_full((M, top - first.shape[1]), -2 ** 62)], 1) if first.shape[1] < top else first
    found = 2 ** 31 - (first & (2 ** 32 - 1))
    value = x.gather(1, found.clamp(0, V - 1))
    real = (found < V) & (first > -2 ** 62) & (value > -math.inf)
    return {"logprob": torch.where(inside, (torch.where(some, d.gather(1, at), -math.inf) - log_total)[:, 0], 0.0),
            "rank": torch.where(inside, rank, -1).int(), "entropy": entropy[:, 0], "lse": lse[:, 0],
            "top_logprob": torch.where(real, (value - torch.where(some, highest, 0.0)) * scale - log_total, -math.inf),
            "top_index": torch.where(real, found, -1)}


_PLAIN = {"rotary": _plain_rotary, "lora": _plain_lora, "logprobs": _plain_logprobs}


# ---------------------------------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The definitions in 64 bits; None for whole numbers (which have to be equal as they are)."""
    st = _inputs(case, seed)
    return {"rotary": _exact_rotary, "lora": _exact_lora, "logprobs": _exact_logprobs}[case["op"]](st)


def _pair_columns(case):
    """The two columns of each pair that turns."""
    i = np.arange(case["rot"] // 2)
    return (2 * i, 2 * i + 1) if case["neighbours"] else (i, i + case["rot"] // 2)


def _exact_rotary(st):
    """Queries in 64 bits.  Codes are whole numbers: those of ties and near ties depend on roundings, which are defined in 32 bits for keys
    (two products and their sum, each rounded) and scales, so that the codes are found there, block by block on the host, and
    valued in 64."""
    case, f32 = st["case"], np.float32
    block, dim = case["block"], case["dim"]
    first, second = _pair_columns(case)
    half = case["rot"] // 2
    q, angles = st["q"].double(), st["table"].double()[st["positions"].long()][:, None, :]
    qr = q.clone()
    qr[..., first] = q[..., first] * angles[..., :half] - q[..., second] * angles[..., half:]
    qr[..., second] = q[..., second] * angles[..., :half] + q[..., first] * angles[..., half:]
    slots, back = st["slots"].cpu().numpy(), st["back"].cpu().numpy()
    cos, sin = np.split(st["table"].cpu().numpy()[st["positions"].cpu().numpy()][:, None, :], 2, 2)
    keys = st["kx"].float().cpu().numpy()
    turned = keys.copy()
    turned[..., first] = keys[..., first] * cos - keys[..., second] * sin
    turned[..., second] = keys[..., second] * cos + keys[..., first] * sin
    blocks = np.unique(np.concatenate([slots, back]) // block)
    at = np.searchsorted(blocks, back // block)
    out = {"q": qr}
    for name, codes, scale, new in (("k", "k", "ks", turned), ("v", "v", "vs", st["vx"].float().cpu().numpy())):
        held = st[codes][torch.tensor(blocks, device=DEV)].cpu().numpy().astype(np.int64)
        sc = st[scale].cpu().numpy().copy()
        t = 0
        while t < len(slots):
            b, begin = int(slots[t] // block), int(slots[t] % block)
            n = 1
            while t + n < len(slots) and slots[t + n] // block == b:
                n += 1
            rows, i = new[t:t + n], int(np.searchsorted(blocks, b))
            for h in range(case["heads"]):
                peak = np.abs(rows[:, h]).max()
                old = sc[b, h] if begin > 0 else f32(0)
                s = max(old, max(f32(peak / f32(127)), f32(TINY)) if peak > 0 else f32(0))
                if begin > 0 and s > old:
                    held[i, h, :begin] = np.rint(held[i, h, :begin].astype(f32) * f32(old / s)).astype(np.int64)
                inv = f32(f32(1) / s) if s > 0 else f32(0)
                held[i, h, begin:begin + n] = np.clip(np.rint(rows[:, h] * inv), -127, 127).astype(np.int64)
                sc[b, h] = s
            t += n
        out[name] = torch.tensor(held[at, :, back % block].astype(np.float64) * sc[back // block].astype(np.float64)[:, :, None])
        out[name + "_scale"] = torch.tensor(sc.astype(np.float64))
    return {name: out[name] for name in ("q", "k", "v", "k_scale", "v_scale")}


def _exact_lora(st):
    y, ids = st["base"].double(), st["ids"].cpu().numpy()
    for a, r in enumerate(st["ranks"]):
        rows = torch.tensor(np.flatnonzero(ids == a), device=DEV)
        if rows.numel():
            y[rows] += st["scale"][a] * ((st["x"][rows].double() @ st["down"][a, :r].double().t()) @ st["up"][a, :, :r].double().t())
    return y


def _exact_logprobs(st):
    x, scale, t, top = st["logits"], st["scale"], st["targets"], st["case"]["top"]
    M, V = x.shape
    out = {"logprob": [], "entropy": [], "lse": [], "top_logprob": []}
    step = max(1, 2 ** 26 // V)
    for i in range(0, M, step):
        z, ti = x[i:i + step].double() * scale, t[i:i + step]
        lse = torch.logsumexp(z, 1, keepdim=True)
        none = lse == -math.inf
        lp = torch.where(none, -math.inf, z - lse)
        inside = (ti >= 0) & (ti < V)
        out["logprob"].append(torch.where(inside, lp.gather(1, ti.clamp(0, V - 1)[:, None])[:, 0], 0.0))
        out["entropy"].append(-torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(1))
        out["lse"].append(lse[:, 0])
        best = lp.topk(min(top, V), 1).values
        out["top_logprob"].append(torch.cat([best, best.new_full((best.shape[0], top - best.shape[1]), -math.inf)], 1))
    out = {name: torch.cat(v) for name, v in out.items()}
    return {"logprob": out["logprob"], "rank": None, "entropy": out["entropy"], "lse": out["lse"], "top_logprob": out["top_logprob"], "top_index": None}


# ----------------------------------------------------------------------------------------------------------------- work
def work(case):
    """Inputs read once, outputs written once, and the products."""
    op = case["op"]
    es = 4 if case["dtype"] == "f32" else 2
    if op == "logprobs":
        M, V = case["rows"], case["vocab"]
        # logits and targets in; four numbers and the alternatives out; a difference, a factor, an exponential and three for the sums
        return {"bytes": M * (V * es + 8 + 16 + 12 * case["top"]), "flops": 6 * M * V}
    if op == "lora":
        ranks, fresh, which = _adapters(case)
        K, N, M = case["K"], case["N"], int(fresh.sum())
        rows = int(fresh[which >= 0].sum())
        used = np.unique(which[(which >= 0) & (fresh > 0)])
        products = int((fresh[which >= 0] * ranks[which[which >= 0]]).sum())
        # rows that have an adapter in, the adapters that are used, base in and Y out
        return {"bytes": es * (rows * K + int(ranks[used].sum()) * (K + N) + 2 * M * N) + 4 * M, "flops": 2 * products * (K + N)}
    ctx, fresh = _lengths(case)
    heads, dim, block, T = case["heads"], case["dim"], case["block"], int(fresh.sum())
    total, begin = ctx + fresh, ctx // block * block
    back = int(np.where(fresh > 0, total - begin, 0).sum())
    touched = int((_ceil(total, block) - ctx // block)[fresh > 0].sum())
    turns = len(np.unique(np.concatenate([np.arange(c, t) for c, t in zip(ctx, total)]))) if T else 0
    # queries in and out, keys and values in, codes out, scales in and out, the angles of the positions that occur; codes in and values out for
    # the tokens that are read back
    return {"bytes": 2 * T * case["q_heads"] * dim * es + 2 * heads * (dim * (T * (es + 1) + back * (1 + es)) + 16 * touched) + 12 * T + 8 * back + 4 * turns * case["rot"],
            "flops": T * (case["q_heads"] + heads) * case["rot"] * 3 + 2 * heads * dim * (3 * T + back)}
