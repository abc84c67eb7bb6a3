"""A layer's self-attention as a serving program runs it, prompts first and then a token of every request at a time:

    plan        blocks and slots for the tokens that arrive                  (abft_kv_plan)
    project     rows x 4-bit weight -> queries, keys and values in one row   (abft_w4_gemv)
    append      keys and values into the 8-bit cache                         (abft_kv_append)
    attend      the new tokens over all that their requests hold             (abft_kv_attention)
    project     rows x 4-bit weight -> the layer's output                    (abft_w4_gemv)

Five launches (six where requests are cut into parts), all on the caller's stream, nothing read back by the host: the host knows the
lengths that it asked for, and with them which blocks of the pool are in use.  Steps of one token each can be recorded as a graph.

`python -m paper_2103_00130_amd.decode_step` runs it on random weights and prints the time of a step, run and replayed.
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


class DecodeLayer:
    """The weights, cache and block tables of one layer for a fixed set of requests."""

    def __init__(self, wqkv: b.W4Weight, wo: b.W4Weight, q_heads: int, heads: int, head_dim: int, requests: int, longest: int, most_rows: int,
                 block_tokens: int = 64, dtype=torch.bfloat16):
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
        self.graph = None

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

    def _launch(self, x, new, free, y, max_new, max_len):
        rows, split = x.shape[0], self.q_heads * self.head_dim
        b.abft_kv_plan(self.ctx, new, self.block, self.table, free, self.seq, self.cu, self.slots[:rows], self.flags, self.taken)
        qkv = self.qkv[:rows]
        b.abft_w4_gemv(x, self.wqkv, qkv)
        q = qkv[:, :split].unflatten(1, (self.q_heads, self.head_dim))
        k, v = qkv[:, split:].unflatten(1, (2, self.heads, self.head_dim)).unbind(1)
        b.abft_kv_append(self.cache, k, v, self.slots[:rows])
        mid = self.mid[:rows]
        b.abft_kv_attention(self.cache, q, self.table, self.seq, self.cu, mid, max_new, max_len, workspace=self.workspace)
        b.abft_w4_gemv(mid.flatten(1), self.wo, y)
        self.ctx.copy_(self.seq)

    def step(self, x, new):
        """x: a row for each new token, those of request 0 first; new: how many each request has (a list).  Returns the rows' output."""
        self._check_rows(x, sum(new))
        first = self._take(new)
        y = torch.empty((x.shape[0], self.wo.N), dtype=x.dtype, device=x.device)
        if x.shape[0]:
            self._launch(x, torch.tensor(new, dtype=torch.int32).to(x.device), self.pool[first:self.used], y, max(new), max(self.lengths))
        return y

    def record(self):
        """Records the step of one token for each request; `replay` runs it."""
        self.x1 = torch.zeros((self.requests, self.wqkv.K), dtype=self.qkv.dtype, device="cuda")
        self.y1 = torch.empty((self.requests, self.wo.N), dtype=self.qkv.dtype, device="cuda")
        self.new1 = torch.ones(self.requests, dtype=torch.int32, device="cuda")
        self.free1 = torch.zeros(self.requests, dtype=torch.int32, device="cuda")   # a step of one token each takes at most so many
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._launch(self.x1, self.new1, self.free1, self.y1, 1, self.longest)

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


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("hidden", 4096), ("q-heads", 32), ("heads", 8), ("head-dim", 128), ("requests", 16), ("prompt", 1000), ("steps", 50), ("block", 64)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args(argv)
    g = torch.Generator("cuda").manual_seed(1)
    wqkv = random_weight((a.q_heads + 2 * a.heads) * a.head_dim, a.hidden, 128, torch.bfloat16, g)
    wo = random_weight(a.hidden, a.q_heads * a.head_dim, 128, torch.bfloat16, g)
    prompts = [max(1, a.prompt * (r + 1) // a.requests) for r in range(a.requests)]
    layer = DecodeLayer(wqkv, wo, a.q_heads, a.heads, a.head_dim, a.requests, a.prompt + 2 * a.steps + 2, max(sum(prompts), a.requests), a.block)
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


if __name__ == "__main__":
    main()
