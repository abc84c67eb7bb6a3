"""A layer's self-attention as a serving program runs it, prompts first and then a token of every request at a time:

    plan        blocks and slots for the tokens that arrive                  (abft_kv_plan)
    project     rows x 4-bit weight -> queries, keys and values in one row   (abft_w4_gemv)
    adapt       what the requests' own low-rank adapters add to it           (abft_lora_gemv, with adapters)
    append      keys and values into the 8-bit cache                         (abft_kv_append, or
                abft_kv_append_rotary with positions, which turns queries and keys on the way)
    attend      the new tokens over all that their requests hold             (abft_kv_attention)
    project     rows x 4-bit weight -> the layer's output                    (abft_w4_gemv)
    adapt       as above

Five launches (six where requests are cut into parts, four more with adapters), all on the caller's stream, nothing read back by the host: the host
knows the lengths that it asked for, and with them which blocks of the pool are in use.  Steps of one token each can be recorded as a graph.
`TokenScores` says what the rows that come out of the last layer mean for given tokens (a 4-bit product and abft_logprobs).

`python -m paper_2103_00130_amd.decode_step` runs it on random weights and prints the time of a step, run and replayed, and of the scores.
"""
from __future__ import annotations

import argparse
import time

import torch

from . import binding as b


def random_weight(n: int, k: int, group: int, dtype, generator) -> b.W4Weight:
    """A weight of random 4-bit codes whose products with normal rows are normal again."""
    codes = torch.randint(0, 256, (n, (k + 1) // 2), dtype=torch.uint8, device="cuda", generator=generator)
    scale = torch.full((n, -(-k // group)), (21.25 * k) ** -0.5, dtype=dtype, device="cuda")   # codes - 7.5 have the variance 21.25
    return b.abft_w4_pack(codes, scale, scale * -7.5, K=k, group=group)


def random_adapters(weight: b.W4Weight, adapters: int, rank: int, dtype, generator) -> b.LoraPool:
    """A pool of random adapters beside a weight, each of whose products is about a tenth of the weight's."""
    pool = b.LoraPool(adapters, weight.K, weight.N, rank, dtype)
    for slot in range(adapters):
        A, B = (torch.randn(shape, device="cuda", generator=generator) for shape in ((rank, weight.K), (weight.N, rank)))
        pool.load(slot, (A * weight.K ** -0.5).to(dtype), (B * rank ** -0.5).to(dtype), 0.1)
    return pool


class DecodeLayer:
    """The weights, cache and block tables of one layer for a fixed set of requests.  rotary: a table of angles (binding.rotary_table) for at least
    `longest` positions, neighbours: which columns turn together; adapters: a pool beside either weight, of which `use` gives a request one."""

    def __init__(self, wqkv: b.W4Weight, wo: b.W4Weight, q_heads: int, heads: int, head_dim: int, requests: int, longest: int, most_rows: int,
                 block_tokens: int = 64, dtype=torch.bfloat16, rotary: torch.Tensor | None = None, neighbours: bool = False,
                 adapters: tuple[b.LoraPool, b.LoraPool] | None = None):
        if rotary is not None:
            if rotary.dim() != 2 or rotary.shape[0] < longest or not 2 <= rotary.shape[1] <= head_dim or rotary.shape[1] % 2 or not rotary.is_contiguous():
                raise ValueError(f"a table of {tuple(rotary.shape)} for requests of up to {longest} tokens and heads of {head_dim} columns: it has a row for each "
                                 "position, for an even number of columns, side by side")
            if not rotary.is_cuda or rotary.dtype != torch.float32:
                raise TypeError("a table of angles is float32 on the device")
        if adapters is not None and len(adapters) != 2:
            raise ValueError(f"{len(adapters)} pools of adapters: a layer has one beside either weight")
        for pool, weight in zip(adapters or (), (wqkv, wo)):
            if (pool.K, pool.N, pool.dtype, pool.adapters) != (weight.K, weight.N, dtype, adapters[0].adapters):
                raise ValueError(f"a pool of {pool.adapters} adapters of {pool.K} to {pool.N} columns in {pool.dtype} beside a weight of {weight.N} x {weight.K}")
        if wqkv.N != (q_heads + 2 * heads) * head_dim or wo.K != q_heads * head_dim:
            raise ValueError(f"weights of {wqkv.N} x {wqkv.K} and {wo.N} x {wo.K} do not fit {q_heads} + 2 x {heads} heads of {head_dim}")
        self.wqkv, self.wo, self.q_heads, self.heads, self.head_dim = wqkv, wo, q_heads, heads, head_dim
        self.requests, self.longest, self.most_rows, self.block = requests, longest, most_rows, block_tokens
        width = -(-longest // block_tokens)
        self.cache = b.KvCache(requests * width, heads, head_dim, block_tokens)
        self.lengths = [0] * requests      # tokens that each request holds, as the host counts them
        self.used = 0                      # blocks of the pool in use
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
        self.pool = torch.arange(requests * width + requests, dtype=torch.int32, device="cuda")   # (a window of `requests` begins anywhere)
        self.table, self.ctx, self.seq, self.cu, self.flags, self.taken = i32(requests, width), i32(requests), i32(requests), i32(requests + 1), i32(requests), i32(1)
        self.slots = torch.zeros(most_rows, dtype=torch.int64, device="cuda")
        self.qkv = torch.empty((most_rows, wqkv.N), dtype=dtype, device="cuda")
        self.mid = torch.empty((most_rows, q_heads, head_dim), dtype=dtype, device="cuda")
        self.workspace = b.KvWorkspace(self.cache, requests, q_heads, max(1, min(longest, most_rows)), longest).tensor
        self.rotary, self.neighbours, self.adapters = rotary, neighbours, adapters
        self.adapter = [-1] * requests     # the slot that each request uses, as the host knows it, and on the device
        self.adapter_of = i32(requests) - 1
        self.lora_workspace = torch.empty(max(b.abft_lora_workspace_bytes(p, most_rows) for p in adapters) // 4, device="cuda") if adapters else None
        self.graph = None

    def use(self, request: int, slot: int):
        """Requests' rows go through the adapter in `slot` from now on (-1: none), replayed steps included."""
        if self.adapters is None or not -1 <= slot < self.adapters[0].adapters:
            raise ValueError(f"no adapter {slot}")
        self.adapter[request] = slot
        self.adapter_of[request] = slot

    def _take(self, new):
        """Checks a step's lengths and counts its tokens and blocks; returns where its blocks begin in the pool."""
        if len(new) != self.requests or any(n < 0 for n in new) or sum(new) > self.most_rows:
            raise ValueError(f"a step takes {self.requests} lengths of {self.most_rows} new tokens in all")
        if any(n + m > self.longest for n, m in zip(self.lengths, new)):
            raise ValueError(f"a request would hold more than {self.longest} tokens")
        first = self.used
        for r, m in enumerate(new):
            self.used += -(-(self.lengths[r] + m) // self.block) - -(-self.lengths[r] // self.block)
            self.lengths[r] += m
        return first

    def _check_rows(self, x, rows):
        # (before anything is counted: a step that is refused leaves the layer as it was)
        if tuple(x.shape) != (rows, self.wqkv.K) or (x.shape[1] > 1 and x.stride(1) != 1):
            raise ValueError(f"x is {tuple(x.shape)}, a step of {rows} new tokens takes {rows} x {self.wqkv.K} with unit column stride")
        if not x.is_cuda or x.dtype != self.qkv.dtype:
            raise TypeError(f"x must be {self.qkv.dtype} on the device")

    def _positions(self, new):
        """Positions of a step's tokens and the adapters of their rows, once their lengths are counted: tensors of the device, None where not wanted."""
        position = adapter = None
        if self.rotary is not None:
            position = torch.cat([torch.arange(n - m, n, dtype=torch.int32) for n, m in zip(self.lengths, new)]).to("cuda")
        if self.adapters is not None:
            adapter = torch.tensor(self.adapter, dtype=torch.int32).repeat_interleave(torch.tensor(new)).to("cuda")
        return position, adapter

    def _launch(self, x, new, free, y, max_new, max_len, position=None, adapter=None):
        rows, split = x.shape[0], self.q_heads * self.head_dim
        b.abft_kv_plan(self.ctx, new, self.block, self.table, free, self.seq, self.cu, self.slots[:rows], self.flags, self.taken)
        qkv = self.qkv[:rows]
        b.abft_w4_gemv(x, self.wqkv, qkv)
        if adapter is not None:
            b.abft_lora_gemv(x, self.adapters[0], adapter, qkv, workspace=self.lora_workspace)
        q = qkv[:, :split].unflatten(1, (self.q_heads, self.head_dim))
        k, v = qkv[:, split:].unflatten(1, (2, self.heads, self.head_dim)).unbind(1)
        if position is None:
            b.abft_kv_append(self.cache, k, v, self.slots[:rows])
        else:
            b.abft_kv_append_rotary(self.cache, q, k, v, self.slots[:rows], position, self.rotary, neighbours=self.neighbours)
        mid = self.mid[:rows]
        b.abft_kv_attention(self.cache, q, self.table, self.seq, self.cu, mid, max_new, max_len, workspace=self.workspace)
        b.abft_w4_gemv(mid.flatten(1), self.wo, y)
        if adapter is not None:
            b.abft_lora_gemv(mid.flatten(1), self.adapters[1], adapter, y, workspace=self.lora_workspace)
        self.ctx.copy_(self.seq)

    def step(self, x, new):
        """x: a row for each new token, those of request 0 first; new: how many each request has (a list).  Returns the rows' output."""
        self._check_rows(x, sum(new))
        held, used = list(self.lengths), self.used
        first = self._take(new)
        try:
            y = torch.empty((x.shape[0], self.wo.N), dtype=x.dtype, device=x.device)
            if x.shape[0]:
                self._launch(x, torch.tensor(new, dtype=torch.int32).to(x.device), self.pool[first:self.used], y, max(new), max(self.lengths),
                             *self._positions(new))
        except Exception:
            # (the device's lengths are the last that a step writes: what it appended before is past every request, and appended anew by the next)
            self.lengths, self.used = held, used
            raise
        return y

    def record(self):
        """Records the step of one token for each request; `replay` runs it."""
        self.x1 = torch.zeros((self.requests, self.wqkv.K), dtype=self.qkv.dtype, device="cuda")
        self.y1 = torch.empty((self.requests, self.wo.N), dtype=self.qkv.dtype, device="cuda")
        self.new1 = torch.ones(self.requests, dtype=torch.int32, device="cuda")
        self.free1 = torch.zeros(self.requests, dtype=torch.int32, device="cuda")   # a step of one token each takes at most so many
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            # (a token of each request is at the position that its request had tokens)
            self._launch(self.x1, self.new1, self.free1, self.y1, 1, self.longest, None if self.rotary is None else self.ctx,
                         None if self.adapters is None else self.adapter_of)

    def replay(self, x):
        """The step of one token for each request, as `record` recorded it; the output is overwritten by the next replay."""
        if self.graph is None:
            raise RuntimeError("nothing is recorded")
        if tuple(x.shape) != self.x1.shape:
            raise ValueError(f"x is {tuple(x.shape)}, a replay takes {tuple(self.x1.shape)}")
        first = self._take([1] * self.requests)
        self.x1.copy_(x)
        self.free1.copy_(self.pool[first:first + self.requests])
        self.graph.replay()
        return self.y1


class TokenScores:
    """What rows of the last layer say about given tokens: a 4-bit weight of a row for each token of the vocabulary, and room for up to most_rows rows."""

    def __init__(self, head: b.W4Weight, most_rows: int, top: int = 0, dtype=torch.bfloat16):
        self.head, self.top = head, top
        new = lambda dt, *shape: torch.empty((most_rows, *shape), dtype=dt, device="cuda")
        self.logits = new(dtype, head.N)
        self.out = {"logprob": new(torch.float32), "rank": new(torch.int32), "entropy": new(torch.float32), "top_logprob": new(torch.float32, top),
                    "top_index": new(torch.int64, top)}
        self.workspace = b.LogprobsWorkspace(most_rows, head.N, top).tensor

    def __call__(self, x, tokens, temperature: float = 1.0):
        """x: rows x hidden; tokens: int64, one for each row.  The results are overwritten by the next call."""
        rows = x.shape[0]
        out = {name: t[:rows] for name, t in self.out.items()}
        b.abft_w4_gemv(x, self.head, self.logits[:rows])
        b.abft_logprobs(self.logits[:rows], tokens, **out, scale=1.0 / temperature, workspace=self.workspace)
        return out


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("hidden", 4096), ("q-heads", 32), ("heads", 8), ("head-dim", 128), ("requests", 16), ("prompt", 1000), ("steps", 50), ("block", 64),
                          ("adapters", 4), ("rank", 16), ("vocab", 32000), ("top", 5)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args(argv)
    g = torch.Generator("cuda").manual_seed(1)
    wqkv = random_weight((a.q_heads + 2 * a.heads) * a.head_dim, a.hidden, 128, torch.bfloat16, g)
    wo = random_weight(a.hidden, a.q_heads * a.head_dim, 128, torch.bfloat16, g)
    longest = a.prompt + 2 * a.steps + 2
    adapters = tuple(random_adapters(w, a.adapters, a.rank, torch.bfloat16, g) for w in (wqkv, wo)) if a.adapters else None
    scores = TokenScores(random_weight(a.vocab, a.hidden, 128, torch.bfloat16, g), a.requests, a.top)
    prompts = [max(1, a.prompt * (r + 1) // a.requests) for r in range(a.requests)]
    layer = DecodeLayer(wqkv, wo, a.q_heads, a.heads, a.head_dim, a.requests, longest, max(sum(prompts), a.requests), a.block,
                        rotary=b.rotary_table(longest, a.head_dim), adapters=adapters)
    for r in range(a.requests if a.adapters else 0):
        layer.use(r, r % (a.adapters + 1) - 1)
    rows = lambda n: torch.randn((n, a.hidden), device="cuda", generator=g).to(torch.bfloat16)
    ones = [1] * a.requests

    def timed(what, n, call):
        torch.cuda.synchronize()
        start = time.perf_counter()
        for _ in range(n):
            call()
        torch.cuda.synchronize()
        print(f"{what}: {(time.perf_counter() - start) / n * 1e6:.1f} us", flush=True)

    x = rows(sum(prompts))
    timed(f"prompts of {prompts[0]} to {prompts[-1]} tokens, {a.requests} requests", 1, lambda: layer.step(x, prompts))
    x = rows(a.requests)
    layer.step(x, ones)
    timed("a token of each, run", a.steps, lambda: layer.step(x, ones))
    layer.record()
    layer.replay(x)
    timed("a token of each, replayed", a.steps, lambda: layer.replay(x))
    tokens = torch.randint(0, a.vocab, (a.requests,), device="cuda", generator=g)
    hidden = layer.y1.clone()
    scores(hidden, tokens)
    timed(f"scores of a token each, {a.top} alternatives", a.steps, lambda: scores(hidden, tokens))


if __name__ == "__main__":
    main()
