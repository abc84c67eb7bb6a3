"""The largest calls of the operators around a decoding step, and numbers at the ends of their types."""
import pytest
import torch

from test_gpu_around_step import b  # noqa: F401 (the fixture)

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
