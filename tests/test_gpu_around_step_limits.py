"""The largest calls of the operators around a decoding step, and numbers at the ends of their types."""
import numpy as np
import pytest
import torch

from test_gpu_around_step import TYPES, b, check_logprobs  # noqa: F401 (b: the fixture)

pytestmark = pytest.mark.gpu


def test_as_many_rows_of_logits_as_a_launch_takes(b):  # noqa: F811
    n = 2 ** 24 - 1
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn((n, 3), device="cuda", generator=g).to(torch.bfloat16)
    targets = torch.randint(0, 3, (n,), device="cuda", generator=g)
    logprob, rank, best = torch.empty(n, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty((n, 1), device="cuda")
    index = torch.empty((n, 1), dtype=torch.int64, device="cuda")
    b.abft_logprobs(x, targets, logprob, rank, top_logprob=best, top_index=index)
    z = x.double() - x.double().logsumexp(1, keepdim=True)
    # a difference, its product with the scale, three exponentials and their sum, a logarithm, a difference: no more than 16 roundings of numbers below 16
    tol = 16 * 16 * 2.0 ** -24
    assert (logprob.double() - z.gather(1, targets[:, None])[:, 0]).abs().max() <= tol
    assert (best.double() - z.max(1, keepdim=True).values).abs().max() <= tol
    mine, lower = x.gather(1, targets[:, None]), torch.arange(3, device="cuda") < targets[:, None]
    assert torch.equal(rank, ((x > mine) | ((x == mine) & lower)).sum(1).int())
    # (of equal ones the first)
    assert torch.equal(index, torch.where(x == x.max(1, keepdim=True).values, torch.arange(3, device="cuda"), 3).amin(1, keepdim=True))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 20000])
def test_logits_at_both_ends_of_their_type(b, dtype, V):  # noqa: F811
    """Differences of logits that binary32 does not hold, whose product with the scale it does."""
    most = torch.finfo(TYPES[dtype]).max
    rng = np.random.default_rng(V)
    x = torch.from_numpy(rng.standard_normal((6, V)).astype(np.float32)).to(TYPES[dtype])
    x[0], x[0, 5] = -most, most
    x[1, 3], x[1, 7] = most, -most
    x[2] = most * torch.from_numpy(rng.uniform(-1, 1, V).astype(np.float32)).to(x.dtype)
    x[3, ::2], x[3, 1::2] = most, -most
    x[4], x[4, 7] = -most, -0.5 * most
    x[5], x[5, 7] = -float("inf"), -most
    for scale in (0.5, 0.01, 1e-30, 2.0 ** -120):
        for target in (3, 5, 7, V - 1):
            check_logprobs(b, x.cuda(), np.full(6, target, np.int64), scale, 8, f"scale {scale}, target {target}")


@pytest.mark.parametrize("K,N", [(64, 2 ** 25), (2 ** 25, 64)])
def test_an_adapter_of_more_elements_than_a_launch_has_threads(b, K, N):  # noqa: F811
    """Rank 128 of K + N = 2^25 + 64 columns: 2^32 + 2^13 elements.  Small whole numbers, whose sums are exact in every type."""
    rank, g = 128, torch.Generator("cuda").manual_seed(2)
    whole = lambda *s: torch.randint(-2, 3, s, dtype=torch.int8, device="cuda", generator=g).to(torch.bfloat16)
    A, B = whole(rank, K), whole(N, rank)
    pool = b.LoraPool(1, K, N, rank)
    pool.load(0, A, B)
    # rows that meet a few columns at both ends and in the middle
    x = torch.zeros((2, K), dtype=torch.bfloat16, device="cuda")
    x[0, [0, K // 2, K - 1]] = 1.0
    x[1, [1, K - 2]] = 2.0
    mid = (A[:, [0, K // 2, K - 1]].float().sum(1), 2.0 * A[:, [1, K - 2]].float().sum(1))
    base = whole(2, N)
    y = torch.empty_like(base)
    b.abft_lora_gemv(x, pool, torch.zeros(2, dtype=torch.int32, device="cuda"), y, base=base, workspace=b.LoraWorkspace(pool, 2).tensor)
    for i in range(2):
        want = base[i].float()
        for n in range(0, N, 2 ** 22):      # (whole numbers below 2^24)
            want[n:n + 2 ** 22] += B[n:n + 2 ** 22].float() @ mid[i]
        assert torch.equal(y[i], want.to(torch.bfloat16))


def test_a_vocabulary_of_more_than_32_bits_is_not_cut_to_them(b):  # noqa: F811
    x = torch.zeros((1, 2 ** 32 + 5), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((1,), 7.0, device="cuda")
    with pytest.raises(ValueError):
        b.abft_logprobs(x, lse=lse)
    assert lse.item() == 7.0


def test_logits_of_more_than_2_to_the_31_elements(b):  # noqa: F811
    M, V, top = 70000, 33000, 3
    x = torch.empty((M, V), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(3))
    targets = torch.arange(M, device="cuda") % V
    results = lambda n: {"logprob": torch.empty(n, device="cuda"), "rank": torch.empty(n, dtype=torch.int32, device="cuda"), "entropy": torch.empty(n, device="cuda"),
                         "top_logprob": torch.empty((n, top), device="cuda"), "top_index": torch.empty((n, top), dtype=torch.int64, device="cuda")}
    whole = results(M)
    b.abft_logprobs(x, targets, **whole)
    for first in (0, 2 ** 31 // V - 600, 2 ** 32 // V // 2 - 10, M - 1100):      # (rows that are not cut either: the same bits)
        rows, some = slice(first, first + 1100), results(1100)
        b.abft_logprobs(x[rows].clone(), targets[rows], **some)
        assert all(torch.equal(some[k], whole[k][rows]) for k in some), first


@pytest.mark.parametrize("K,N", [(8_000_000, 16), (16, 8_000_000)])
def test_rows_of_adapters_of_more_than_2_to_the_31_elements(b, K, N):  # noqa: F811
    """Whole numbers, whose sums are exact however they are cut."""
    M, rank, g = 300, 4, torch.Generator("cuda").manual_seed(4)
    whole = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").uniform_(-1.49, 1.49, generator=g).round_()
    x, base, pool = whole(M, K), whole(M, N), b.LoraPool(2, K, N, rank)
    for slot in range(2):
        A, B = whole(rank, K), whole(N, rank)
        A[:, 64:] *= (torch.rand(max(K - 64, 0), device="cuda", generator=g) < 1e-5).to(A.dtype)      # (sums below 2^8, which bfloat16 holds)
        pool.load(slot, A, B)
    ids = (torch.arange(M, device="cuda") % 3 - 1).int()
    y = torch.empty_like(base)
    b.abft_lora_gemv(x, pool, ids, y, base=base, workspace=b.LoraWorkspace(pool, M).tensor)
    for first in (0, 260, M - 20):
        rows = slice(first, first + 20)
        some = base[rows].clone()
        b.abft_lora_gemv(x[rows].clone(), pool, ids[rows].clone(), some, workspace=b.LoraWorkspace(pool, 20).tensor)
        assert torch.equal(some, y[rows]) and not torch.equal(some, base[rows]), first


def test_queries_of_more_than_2_to_the_31_elements(b):  # noqa: F811
    T, q_heads, dim, block = 70000, 256, 128, 64
    q = torch.empty((T, q_heads, dim), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(5))
    kv = torch.randn((T, 2, 1, dim), device="cuda").to(torch.bfloat16)
    table, c = b.rotary_table(1000, dim), b.KvCache(T // block + 1, 1, dim, block)
    at = torch.arange(T, device="cuda")
    slots, pos = at, (at % 1000).int()
    turned = torch.empty_like(q)
    b.abft_kv_append_rotary(c, q, kv[:, 0], kv[:, 1], slots, pos, table, QR=turned)
    for first in (0, 65536 - 64, T // block * block - 640):
        rows, d = slice(first, first + 640), b.KvCache(10, 1, dim, block)
        some = q[rows].clone()
        b.abft_kv_append_rotary(d, some, kv[rows, 0], kv[rows, 1], at[:640], pos[rows], table)
        assert torch.equal(some, turned[rows])
        for one, two in zip(d.codes(), c.codes()):
            assert torch.equal(one, two[first // block:first // block + 10])
    b.abft_kv_append_rotary(c, q, kv[:, 0], kv[:, 1], slots, pos, table)      # in place
    assert torch.equal(q, turned)
