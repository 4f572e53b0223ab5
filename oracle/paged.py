"""Oracle of the paged cache in 8 bits and of the operators on pages: the e4m3
codes by their definition, a page's power of two, appends token by token, and page
tables by loops over rows.  Shares no code with the CUDA path."""
from __future__ import annotations

import math

import numpy as np

# the 127 magnitudes of e4m3: 4 bits of exponent (bias 7), 3 of mantissa, code 127 is NaN
MAGNITUDES = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])
RANGE = {"bf16": (-110, 119), "f16": (-15, 7)}


def decode(codes):
    """The numbers that codes (uint8) stand for."""
    c = np.asarray(codes, np.int64)
    mag = np.where((c & 127) == 127, np.nan, MAGNITUDES[np.minimum(c & 127, 126)])
    return np.where(c & 128, -mag, mag)


def encode(x):
    """The nearest code, ties to the even one, at most 448 in magnitude; NaN (0x7f) for what is not finite."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    a = np.minimum(np.abs(np.where(fine, x, 0.0)), 448.0)
    lo = np.clip(np.searchsorted(MAGNITUDES, a, side="right") - 1, 0, 126)
    hi = np.minimum(lo + 1, 126)
    below, above = a - MAGNITUDES[lo], MAGNITUDES[hi] - a
    code = np.where((above < below) | ((above == below) & (lo % 2 == 1)), hi, lo)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(fine, code, 127).astype(np.uint8)


def exponent(x, lo, hi):
    """Least e in [lo, hi] with max |x| <= 448 * 2^e, of the finite numbers."""
    x = np.abs(np.asarray(x, np.float64))
    top = x[np.isfinite(x)].max(initial=0.0)
    e = lo
    while e < hi and top > math.ldexp(448.0, e):
        e += 1
    return e


def append(codes, exps, x, first, table_row, page, lo, hi):
    """x [n, H, D], a sequence's positions first .. first + n - 1, into codes
    [P, H, page, D] (uint8) and exps [P, H], in place."""
    x = np.asarray(x, np.float64)
    n = len(x)
    for i in range(first // page, (first + n - 1) // page + 1 if n else 0):
        a, b = max(first, i * page), min(first + n, (i + 1) * page)
        pg = int(table_row[i])
        for h in range(x.shape[1]):
            part = x[a - first:b - first, h]
            e = exponent(part, lo, hi)
            s0, s1 = a - i * page, b - i * page
            if s0 > 0:
                old = int(exps[pg, h])
                e = max(e, old)
                if e > old:
                    codes[pg, h, :s0] = encode(np.ldexp(decode(codes[pg, h, :s0]), old - e))
            exps[pg, h] = e
            codes[pg, h, s0:s1] = encode(np.ldexp(part, -e))


def values(codes, exps):
    """What pages [P, H, page, D] hold."""
    return np.ldexp(decode(codes), np.asarray(exps, np.int64)[..., None, None])


def fork(refs, table, lengths, parents, after, width, page):
    """(refs, table, copies [(from, to)], short): rows that go on from the table's;
    short: entries that no free page was left for."""
    refs, table = [int(r) for r in refs], [[int(x) for x in row] for row in table]
    pages = lambda t: (t + page - 1) // page  # noqa: E731
    rows = []
    for i, p in enumerate(parents):
        held = int(lengths[p]) if p >= 0 else 0
        end = int(after[i]) if after is not None else held
        rows.append((int(p), min(held, end), end))
    free = [x for x, r in enumerate(refs) if r == 0]
    out, copies, short = [], [], 0
    for i, (p, kept, end) in enumerate(rows):
        row = table[p][:pages(kept)] if p >= 0 else []
        if kept % page:
            last = len(row) - 1
            own = refs[row[last]] == 1
            for j, (q, k, _) in enumerate(rows):
                if j != i and q == p and pages(k) > last:
                    full = k >= (last + 1) * page
                    own = own and not full and j > i
            if not own:
                to = free.pop(0) if free else -1
                short += to < 0
                if to >= 0:
                    copies.append((row[last], to))
                row[last] = to
        while len(row) < pages(end):
            row.append(free.pop(0) if free else -1)
            short += row[-1] < 0
        out.append(row + [-1] * (width - len(row)))
    new = list(refs)
    for b, row in enumerate(table):
        for x in row[:pages(int(lengths[b]))]:
            new[x] -= 1
    for row in out:
        for x in row:
            if x >= 0:
                new[x] += 1
    return np.array(new), np.array(out).reshape(len(rows), width), copies, short


def compact(refs, table, lengths, page):
    """(refs, table, where, moves [(from, to)])."""
    n, used = len(refs), [x for x, r in enumerate(refs) if r > 0]
    u = len(used)
    moves = list(zip([x for x in used if x >= u], [x for x in range(u) if refs[x] == 0]))
    where = [x if refs[x] > 0 else -1 for x in range(n)]
    for a, b in moves:
        where[a] = b
    new = [0] * n
    for x in used:
        new[where[x]] = int(refs[x])
    out = [[where[int(x)] if j < (int(lengths[b]) + page - 1) // page else -1 for j, x in enumerate(row)]
           for b, row in enumerate(table)]
    return np.array(new), np.array(out).reshape(np.asarray(table).shape), np.array(where), moves
