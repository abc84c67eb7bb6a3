"""Log probabilities of prompts: more rows than are cut into parts, of many batches each, whose bars rise as a row is gone through.  Rows of all kinds lie among
them; some of each are checked against the oracle, and all against the same rows alone, which are cut."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as o
from test_gpu_around_step import TYPES, b, dev, f64, run_logprobs, within  # noqa: F401 (b: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V,top", [(40001, 20), (33000, 64), (50000, 0), (70000, 1)])
def test_logprobs_of_prompts(b, dtype, V, top):  # noqa: F811
    M, kinds, inf = 1040, 8, float("inf")
    g = torch.Generator("cuda").manual_seed(V + top)
    x = torch.randn((M, V), device="cuda", generator=g) * 2
    kind = torch.arange(M, device="cuda") % kinds
    rising = torch.linspace(-6, 6, V, device="cuda")
    x[kind == 1] = rising                                             # every logit reaches the bar (with ties in 16 bits)
    x[kind == 2] = -rising
    x[kind == 3] = x[kind == 3].round()                               # many ties
    x[kind == 4] = x[kind == 4].masked_fill(torch.rand((int((kind == 4).sum()), V), device="cuda", generator=g) < 0.999, -inf)
    x[kind == 5, : V - 30] = -inf                                     # all that there is at the end
    x[kind == 6] = 1.5                                                # all the same
    x[kind == 7, 30:] -= 12.0                                         # the best at the beginning
    x = x.to(TYPES[dtype])
    rng = np.random.default_rng(V)
    targets = rng.integers(0, V, M).astype(np.int64)
    targets[rng.random(M) < 0.1] = -1
    targets[rng.random(M) < 0.3] = V - 5
    got = run_logprobs(b, x, targets, 1.25, top)
    some = np.concatenate([np.arange(kinds), rng.integers(0, M, 16)])
    want = o.logprobs(f64(x[dev(some)]), targets[some], 1.25, top)
    assert np.array_equal(got["rank"][some], want["rank"]) and np.array_equal(got["top_index"][some], want["top_index"])
    for name, tol in (("logprob", "logprob_tol"), ("entropy", "entropy_tol"), ("lse", "lse_tol"), ("top_logprob", "top_tol")):
        within(got[name][some].astype(np.float64), want[name], want[tol], name)
    # fewer rows are cut into parts: whole numbers equal, and the rest within both errors
    for first in range(0, M, 208):
        rows = slice(first, first + 208)
        part = run_logprobs(b, x[rows], targets[rows], 1.25, top)
        assert np.array_equal(part["rank"], got["rank"][rows]) and np.array_equal(part["top_index"], got["top_index"][rows])
    again = run_logprobs(b, x, targets, 1.25, top)
    assert all(np.array_equal(again[k], got[k], equal_nan=True) for k in got)
