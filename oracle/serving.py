"""Oracle of the serving operators, in float64: rotary positions with several
axes, the page table, and causal attention of the last queries of a sequence
with an optional window.  Loops over sequences and heads; shares no code with
the CUDA path."""
from __future__ import annotations

import numpy as np


def rotary(x, pos, inv_freq, axis, adjacent=False, factor=1.0):
    """x [N, H, D] rotated to pos [axes, N]: pair i of channels turns by
    pos[axis[i]] * inv_freq[i]."""
    x = np.asarray(x, np.float64)
    inv_freq, axis = np.asarray(inv_freq, np.float64), np.asarray(axis)
    n = len(inv_freq)
    ang = np.asarray(pos, np.float64)[axis].T * inv_freq          # [N, n]
    c, s = factor * np.cos(ang)[:, None], factor * np.sin(ang)[:, None]
    first = 2 * np.arange(n) if adjacent else np.arange(n)
    second = first + (1 if adjacent else n)
    out = x.copy()
    out[..., first] = x[..., first] * c - x[..., second] * s
    out[..., second] = x[..., second] * c + x[..., first] * s
    return out


def place(t, table_row, page):
    """(page, slot) of position t of a sequence with this row of the table."""
    return int(table_row[t // page]), t % page


def from_pages(pool, table_row, n, page):
    """The first n positions [H, n, D] of a sequence from a pool [P, H, page, D]."""
    pool = np.asarray(pool, np.float64)
    t = np.arange(n)
    rows = np.asarray(table_row)[t // page]
    return np.transpose(pool[rows, :, t % page], (1, 0, 2))


def attend(q, k, v, scale, window=0):
    """q [n, Hq, D], the queries of the last n of the positions of k, v
    [Hkv, t, D].  Returns the outputs and, for error bounds, sum_t p_t |v_t|
    per channel, sum_t |v_t| over the positions seen and the largest
    scale * sum_i |q_i k_i| of each row."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    n, hq, d = q.shape
    hkv, t, _ = k.shape
    out = np.zeros((n, hq, d))
    mass, plain, span = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq))
    for i in range(n):
        p = t - n + i
        if p < 0:
            continue
        lo = max(0, p - window + 1) if window else 0
        for h in range(hq):
            kk, vv = k[h // (hq // hkv), lo:p + 1], v[h // (hq // hkv), lo:p + 1]
            with np.errstate(invalid="ignore", over="ignore"):
                x = scale * (kk @ q[i, h])
                w = np.exp(x - x.max())
                w /= w.sum()
                out[i, h] = w @ vv
                mass[i, h] = w @ np.abs(vv)
                plain[i, h] = np.abs(vv).sum(0)
                span[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, mass, plain, span


def attend_bound(out, mass, plain, span, d, t, u, smallest):
    """How far a kernel may be off: binary32 scores (d products summed, each
    step 2^-23 of the row's sum of magnitudes, which also enters the weights'
    sum), weights by a base-2 exponential good to 2^-21, rounded to the stored
    type (u, half a step; below its normal range `smallest`, half its last step
    there), products summed over t positions, the result rounded (u)."""
    soft = 2 * (d + 4) * 2.0 ** -23 * span[..., None] + 2.0 ** -20 + 2 * (t + 8) * 2.0 ** -23
    with np.errstate(invalid="ignore"):  # infinite results
        return u * np.abs(out) * (1 + u) + (1 + 2 * u) * (u + soft) * mass + smallest * plain + 2.0 ** -126
