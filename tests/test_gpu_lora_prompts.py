"""Adapters as prompts meet them: rows of several hundred tokens and more, one workgroup to the adapters of a tile, several blocks of columns to a wavefront, whose
loads run ahead of its stores; in place too.  Against the definition in 64 bits, within the error that step_oracle derives."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as o
from oracle.decode_oracle import TINY, UNIT
from test_gpu_around_step import TYPES, b, dev, f64, values  # noqa: F401 (b: the fixture)

pytestmark = pytest.mark.gpu


def lora64(X, adapters, ids, base, dtype):
    """step_oracle.lora, the rows of an adapter together, wherever the tensors lie."""
    X, Y = X.double(), base.double().clone()
    err = torch.zeros_like(Y)
    for a, adapter in enumerate(adapters):
        rows = torch.from_numpy(np.flatnonzero(ids == a)).to(X.device)
        if adapter is None or not len(rows) or adapter[0].shape[0] == 0:
            continue
        A, B, scale = adapter[0].double(), adapter[1].double(), float(np.float32(adapter[2]))
        x = X[rows]
        mid = x @ A.t()
        mid_err = (A.shape[1] + 16) * 2.0 ** -23 * (x.abs() @ A.abs().t())
        d_err = mid_err @ B.abs().t() + (B.shape[1] + 16) * 2.0 ** -23 * ((mid.abs() + mid_err) @ B.abs().t())
        Y[rows] += scale * (mid @ B.t())
        err[rows] = abs(scale) * d_err + 2.0 ** -23 * Y[rows].abs()
    return Y, err + UNIT[dtype] * Y.abs() + TINY[dtype]


def close(got, want, tol, what):
    off = ~((got.double() - want).abs() <= tol)
    assert not off.any(), f"{what}: {int(off.sum())} of {off.numel()} beyond the bound, first {off.nonzero()[0].tolist()}: {got[off][0].item()!r} for {want[off][0].item()!r} +- {tol[off][0].item():.3g}"


def test_rows_of_an_adapter_together_are_the_oracle():
    rng = np.random.default_rng(1)
    X, base, ids = rng.standard_normal((9, 12)), rng.standard_normal((9, 7)), np.array([0, 2, -1, 1, 0, 3, 9, 2, 0])
    adapters = [(rng.standard_normal((r, 12)), rng.standard_normal((7, r)), 0.7) for r in (3, 1, 0)] + [None]
    want, tol = o.lora(X, adapters, ids, base, "bf16")
    got, bound = lora64(torch.from_numpy(X), [a and (torch.from_numpy(a[0]), torch.from_numpy(a[1]), a[2]) for a in adapters], ids, torch.from_numpy(base), "bf16")
    assert np.allclose(got.numpy(), want, rtol=1e-13) and np.allclose(bound.numpy(), tol, rtol=1e-12)


# (rows, K, N, ranks, the pool's, at least so many blocks of 64 columns to a wavefront in 16 and in 32 bits)
PROMPTS = [(530, 264, 20001, [8, 16, 5], 16, 3, 3), (1100, 2100, 9001, [40, 7], 48, 3, 9), (4000, 72, 4099, [32, 20, 1, 0], 32, 4, 4), (530, 500, 5000, [128, 72, 40], 128, 1, 3),
           (4300, 40, 1500, [72, 128, 16], 128, 2, 6), (600, 1500, 1500, [40, 72, 128], 128, 1, 1), (300, 1030, 4000, [16, 2, 16, 9], 16, 3, 3), (128, 200, 6003, [64, 17], 64, 3, 12),
           (512, 33, 16500, [24, 31], 31, 3, 3), (16390, 64, 333, [16, 3], 16, 2, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,K,N,ranks,max_rank,blocks16,blocks32", PROMPTS)
def test_lora_of_prompts(b, dtype, M, K, N, ranks, max_rank, blocks16, blocks32):  # noqa: F811
    rng = np.random.default_rng(M + K + N)
    pool = b.LoraPool(len(ranks), K, N, max_rank, TYPES[dtype])
    pool.down.fill_(float("nan"))
    pool.up.fill_(float("nan"))
    plain = []
    for a, r in enumerate(ranks):
        A, B, scale = values(rng, (max(r, 1), K), dtype)[:r], values(rng, (N, max(r, 1)), dtype)[:, :r], float(rng.uniform(0.2, 2))
        pool.load(a, A if r else None, B if r else None, scale)
        plain.append((A, B, scale))
    for turn in range(3):
        if turn == 0:        # prompts that begin anywhere, some without an adapter
            cuts = np.sort(rng.choice(np.arange(1, M), min(9, M - 1), replace=False))
            ids = np.repeat(rng.integers(-1, len(ranks), len(cuts) + 1), np.diff(np.concatenate([[0], cuts, [M]])))
        elif turn == 1:      # in no order, with rows that have none or one that does not exist
            ids = rng.choice(list(range(len(ranks))) + [-1, len(ranks), 2 ** 31 - 1], M)
        else:
            ids = np.full(M, int(np.argmax(ranks)))
        ids = ids.astype(np.int32)
        off = turn % 2       # rows further apart than they are long, off any wide alignment
        x = values(rng, (M, K + 5 * off), dtype)[:, off:K + off]
        base, y = values(rng, (M + 1, N + 3 * off), dtype), torch.full((M + 1, N + 2 * off), 7.0, dtype=TYPES[dtype], device="cuda")
        ws = b.LoraWorkspace(pool, M).tensor
        ws.fill_(float("nan"))
        b.abft_lora_gemv(x, pool, dev(ids), y[:M, off:N + off], base=base[:M, :N], workspace=ws)
        close(y[:M, off:N + off], *lora64(x, plain, ids, base[:M, :N], dtype), f"turn {turn}")
        assert (y[M:] == 7.0).all() and (y[:, :off] == 7.0).all() and (y[:, N + off:] == 7.0).all()
        z = base.clone()     # in place: the same bits
        b.abft_lora_gemv(x, pool, dev(ids), z[:M, :N], workspace=ws)
        assert torch.equal(z[:M, :N], y[:M, off:N + off]) and torch.equal(z[M:], base[M:]) and torch.equal(z[:, N:], base[:, N:])
        again = torch.empty_like(y)
        b.abft_lora_gemv(x, pool, dev(ids), again[:M, off:N + off], base=base[:M, :N], workspace=ws)
        assert torch.equal(again[:M, off:N + off], y[:M, off:N + off])
