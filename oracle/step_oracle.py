"""Oracle of the operators around a decoding step's products and attention (abft_kv_append_rotary in include/abft_eb.h, abft_lora_gemv and
abft_logprobs in include/abft_gemm.h): plain numpy, 64-bit floats except where the definition fixes 32 (the rotation).  Test infrastructure
only.

Next to each value that depends on rounding stands the error that its kernel may make, derived here from the header's statement of the
arithmetic, not from what a kernel gave."""
from __future__ import annotations

import numpy as np

from .decode_oracle import TINY, UNIT


# ------------------------------------------------------------------------------------------------------------------ rotation
def rotate(x, table, positions, neighbours):
    """x [T][heads][dim] (float32) turned: binary32, one rounding after each product and each sum."""
    x = x.astype(np.float32)
    out = x.copy()
    half = table.shape[1] // 2
    for t, pos in enumerate(positions):
        if not 0 <= pos < len(table):
            continue
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if neighbours else (i, half + i)
            c, s = np.float32(table[pos, i]), np.float32(table[pos, half + i])
            with np.errstate(invalid="ignore", over="ignore"):
                out[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
                out[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return out


# ------------------------------------------------------------------------------------------------------------------ adapters
def lora(X, adapters, ids, base, dtype):
    """(Y, tolerance); adapters: (A [rank][K], B [N][rank], scale) of each slot, or None.  Every addition in binary32 errs by at most 2^-23 of
    the magnitudes added so far (2^-24 rounded to nearest; the matrix cores may cut instead), and so does a binary32 product."""
    X, Y = X.astype(np.float64), base.astype(np.float64).copy()
    err = np.zeros_like(Y)
    for m, a in enumerate(ids):
        if not 0 <= a < len(adapters) or adapters[a] is None or adapters[a][0].shape[0] == 0:
            continue
        A, B, scale = adapters[a]
        A, B, scale = A.astype(np.float64), B.astype(np.float64), float(np.float32(scale))
        mid = A @ X[m]
        mid_err = (A.shape[1] + 16) * 2.0 ** -23 * (np.abs(A) @ np.abs(X[m]))
        d = B @ mid
        d_err = np.abs(B) @ mid_err + (B.shape[1] + 16) * 2.0 ** -23 * (np.abs(B) @ (np.abs(mid) + mid_err))
        Y[m] += scale * d
        err[m] = abs(scale) * d_err + 2.0 ** -23 * np.abs(Y[m])
    return Y, err + UNIT[dtype] * np.abs(Y) + TINY[dtype]


# --------------------------------------------------------------------------------------------------------- log probabilities
def logprobs(x, targets, scale, top):
    """x [rows][vocab] (float64, as the type holds them).  A dict of (value, tolerance), or whole numbers alone.

    Errors.  t = scale log2(e) (x - m) errs by three roundings, 2^t by as much times ln 2 of itself and by its last place; a sum of V terms is taken by
    at least 256 lanes in turns of eight and joined in some twenty steps, each of which may also bring it to a larger m (another factor): its terms err by
    2^-23 for each of at most V / 256 + 100 steps, and by 2^-21 of |t|.  The logarithm by two last places."""
    scale = float(np.float32(scale))
    M, V = x.shape
    out = {k: np.zeros(M) for k in ("logprob", "entropy", "lse", "logprob_tol", "entropy_tol", "lse_tol")}
    out["rank"] = np.full(M, -1, np.int32)
    out["top_logprob"], out["top_tol"], out["top_index"] = np.full((M, top), -np.inf), np.zeros((M, top)), np.full((M, top), -1, np.int64)
    index = np.arange(V)
    for r in range(M):
        t = int(targets[r]) if targets is not None else -1
        inside = 0 <= t < V
        if np.isnan(x[r]).any() or (x[r] == np.inf).any():
            out["logprob"][r] = np.nan if inside else 0.0
            out["entropy"][r] = out["lse"][r] = np.nan
            out["top_logprob"][r] = np.nan
            continue
        if inside:
            out["rank"][r] = np.count_nonzero((x[r] > x[r, t]) | ((x[r] == x[r, t]) & (index < t)))
        if not (x[r] > -np.inf).any():
            out["logprob"][r], out["lse"][r] = -np.inf if inside else 0.0, -np.inf
            continue
        live = x[r] > -np.inf
        m = x[r].max()
        d = scale * (x[r][live] - m)
        e = np.exp(d)
        s = e.sum()
        p, u = e / s, np.abs(d) / np.log(2)
        steps = 2.0 ** -23 * (V / 256 + 100)
        rel = steps + 2.0 ** -21 * (p @ u)
        ln_err = rel + 2.0 ** -22 * (1 + abs(np.log(s)))
        out["lse"][r], out["lse_tol"][r] = scale * m + np.log(s), ln_err + 2.0 ** -22 * abs(scale * m)
        out["entropy"][r] = np.log(s) - p @ d
        out["entropy_tol"][r] = ln_err + (p @ u) * (steps + rel + 2.0 ** -21) + 2.0 ** -21 * (p @ u ** 2) + 2.0 ** -22 * (1 + out["entropy"][r])
        of = lambda v: scale * (v - m) - np.log(s)
        tol = lambda v: ln_err + 2.0 ** -22 * abs(scale * (v - m)) + 2.0 ** -23 * abs(of(v))
        if inside:
            out["logprob"][r] = of(x[r, t])
            out["logprob_tol"][r] = tol(x[r, t]) if live[t] else 0.0
        order = np.lexsort((index, -(x[r] + 0.0)))[:top]
        order = order[live[order]]
        out["top_index"][r, :len(order)] = order
        out["top_logprob"][r, :len(order)] = of(x[r, order])
        out["top_tol"][r, :len(order)] = tol(x[r, order])
    return out
