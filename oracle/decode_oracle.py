"""Oracle of the decoding-step operators (abft_w4_* in include/abft_gemm.h, abft_kv_* in include/abft_eb.h): plain numpy, loops where
the definition has them, 64-bit floats except where the definition fixes 32 (scales and codes of the cache).  Test infrastructure only.

Next to each value that depends on rounding stands the error that its kernel may make, derived here from the header's statement of the
arithmetic, not from what a kernel gave."""
from __future__ import annotations

import numpy as np

# unit roundoff of the types that results are rounded to
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # (bfloat16: half of 2^-7)
# the smallest step of a type, for results near zero
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}


# ------------------------------------------------------------------------------------------------------------- 4-bit weights
def unpack_codes(W: np.ndarray, K: int) -> np.ndarray:
    """[N][K] codes from bytes of two, the even column in the low half."""
    out = np.empty((W.shape[0], 2 * W.shape[1]), dtype=np.int64)
    out[:, 0::2] = W & 15
    out[:, 1::2] = W >> 4
    return out[:, :K]


def w4_product(X, W, scale, bias, group, dtype):
    """(Y, tolerance) of X W^T.  A group's sum of x * (16 + code) and its sum of x, each of up to `group` products, and a sum over the
    groups: every addition in binary32 errs by at most 2^-23 of the magnitudes added so far (2^-24 rounded to nearest; the matrix
    cores may cut instead), twice over for the products with scale and shift."""
    X = X.astype(np.float64)
    K = X.shape[1]
    codes = unpack_codes(W, K).astype(np.float64)
    g = np.arange(K) // group
    s = scale.astype(np.float64)[:, g]
    b = -8.0 * s if bias is None else bias.astype(np.float64)[:, g]
    Y = X @ (s * codes + b).T
    size = np.abs(X) @ (np.abs(s) * (16 + codes) + np.abs(b - 16 * s)).T
    steps = group + scale.shape[1] + 8
    return Y, steps * 2.0 ** -23 * size + UNIT[dtype] * np.abs(Y) + TINY[dtype]


# -------------------------------------------------------------------------------------------------------- tables and slots
def plan(ctx_len, new_len, block, table, free, n_slots):
    """abft_kv_plan request by request; the table is extended in place."""
    R, width = len(ctx_len), table.shape[1]
    seq, cu, slots, flags = [], [0], [], []
    rows = need_sum = taken = 0
    for r in range(R):
        ctx, new = max(int(ctx_len[r]), 0), max(int(new_len[r]), 0)
        why = 8 if ctx_len[r] < 0 or new_len[r] < 0 else 0
        have, want = -(-ctx // block), -(-(ctx + new) // block)
        rows += new
        refused = 0
        if want > width:
            refused |= 2
        if rows > n_slots:
            refused |= 4
        if not refused and want > have:
            if need_sum + want - have > len(free):
                refused |= 1
            else:
                taken = need_sum + want - have
                table[r, have:want] = free[need_sum:taken]
            need_sum += want - have
        flags.append(why | refused)
        seq.append(ctx if refused else ctx + new)
        for p in range(ctx, ctx + new):
            if len(slots) < n_slots:
                slots.append(-1 if refused else int(table[r, p // block]) * block + p % block)
        cu.append(min(rows, n_slots))
    slots += [-1] * (n_slots - len(slots))
    i32 = np.int32
    return np.array(seq, i32), np.array(cu, i32), np.array(slots, np.int64), np.array(flags, i32), taken


# -------------------------------------------------------------------------------------------------------------------- cache
def append(codes, scale, x, slots):
    """New rows x [T][heads][dim] (float32) into codes [blocks][heads][block][dim] and scale [blocks][heads], in place."""
    f = np.float32
    n_blocks, heads, block, _ = codes.shape
    t = 0
    while t < len(slots):
        s0 = int(slots[t])
        if not 0 <= s0 < n_blocks * block:
            t += 1
            continue
        n = 1
        while t + n < len(slots) and slots[t + n] == s0 + n and (s0 + n) // block == s0 // block:
            n += 1
        b, first = s0 // block, s0 % block
        for h in range(heads):
            v = x[t:t + n, h].astype(f)
            finite = np.abs(v[np.isfinite(v)])
            peak = finite.max() if finite.size else f(0)
            s = scale[b, h] if first > 0 else f(0)
            old = s
            if peak > 0:
                s = max(s, max(f(peak / f(127)), f(2.0 ** -126)))
            if first > 0 and s > old:
                codes[b, h, :first] = np.clip(np.rint(codes[b, h, :first].astype(f) * f(old / s)), -127, 127)
            with np.errstate(over="ignore", invalid="ignore"):
                y = np.rint(v * (f(f(1) / s) if s > 0 else f(0)))
            codes[b, h, first:first + n] = np.clip(np.nan_to_num(y, nan=0.0, posinf=127, neginf=-127), -127, 127)
            scale[b, h] = s
        t += n


def read(codes, scale, slots):
    """[T][heads][dim] in 64 bits."""
    n_blocks, heads, block, dim = codes.shape
    out = np.zeros((len(slots), heads, dim))
    for t, s in enumerate(slots):
        if 0 <= s < n_blocks * block:
            out[t] = codes[s // block, :, s % block].astype(np.float64) * scale[s // block].astype(np.float64)[:, None]
    return out


# ---------------------------------------------------------------------------------------------------------------- attention
def attention(q, k_codes, v_codes, k_scale, v_scale, table, seq_len, cu_new, scale, dtype):
    """(O, tolerance, lse, tolerance of lse) for q [rows][q_heads][dim].

    Errors.  Q as a fixed-point number of 2^k steps: half a step of its row's largest element / one for each element, one being 127 *
    256 (16-bit types) or 63 * 65536; a score thus errs by half a step times the sum of |K|, and by a few roundings of binary32.  A
    numerator errs relatively by that (and by exp2's last place), and absolutely by half a step of the largest numerator times value
    scale of its 64 tokens.  Sums in binary32 err by 2^-23 for each tile that is added."""
    rows, q_heads, dim = q.shape
    n_blocks, heads, block, _ = k_codes.shape
    group = q_heads // heads
    q_one, p_one = (63 * 65536.0, 127 * 65536.0) if dtype == "f32" else (127 * 256.0, 127 * 256.0)
    O, tol = np.zeros(q.shape), np.zeros(q.shape)
    lse, lse_tol = np.full((rows, q_heads), -np.inf), np.zeros((rows, q_heads))
    for r in range(len(seq_len)):
        length, c0, c1 = max(int(seq_len[r]), 0), int(cu_new[r]), int(cu_new[r + 1])
        pos = np.arange(length)
        ids = table[r, pos // block].astype(np.int64)
        good = (ids >= 0) & (ids < n_blocks)
        ids = np.where(good, ids, 0)
        off = pos % block
        tiles = pos // 64
        for t in range(c0, c1):
            sees = length - (c1 - c0) + (t - c0) + 1
            seen = good[:max(sees, 0)]
            if not seen.any():
                continue
            for i in range(q_heads):
                h = i // group
                sel = np.flatnonzero(seen)
                kc, vc = k_codes[ids[sel], h, off[sel]].astype(np.float64), v_codes[ids[sel], h, off[sel]].astype(np.float64)
                ks, vs = k_scale[ids[sel], h].astype(np.float64), v_scale[ids[sel], h].astype(np.float64)
                x = q[t, i].astype(np.float64)
                z = (kc @ x) * ks * scale
                dz = np.abs(kc).sum(1) * ks * abs(scale) * (0.5 / q_one) * np.abs(x).max() + 2.0 ** -21 * (1 + np.abs(z).max() + np.abs(z))
                top = z.max()
                p = np.exp(z - top)
                total = p.sum()
                w = p / total
                v = vc * vs[:, None]
                O[t, i] = w @ v
                lse[t, i] = top + np.log(total)
                size = w @ np.abs(v)
                wv = w * vs
                step = np.zeros(dim)
                n_tiles = 0
                for g in np.unique(tiles[sel]):
                    m = tiles[sel] == g
                    step += wv[m].max() * np.abs(vc[m]).sum(0) * (0.5 / p_one)
                    n_tiles += 1
                rel = 2 * dz.max() + (8 + 2 * n_tiles) * 2.0 ** -23
                tol[t, i] = size * rel + step * (1 + rel) + UNIT[dtype] * np.abs(O[t, i]) + TINY[dtype]
                lse_tol[t, i] = rel + 2.0 ** -22 * (1 + abs(lse[t, i]))
    return O, tol, lse, lse_tol
