"""The oracle of the paged cache in 8 bits and of the operators on pages against
torch's float8, brute force and worked examples."""
import math

import numpy as np
import pytest
import torch

from oracle import paged


def test_codes_are_torch_float8():
    c = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = c.view(torch.float8_e4m3fn).double().numpy()
    got = paged.decode(c.numpy())
    np.testing.assert_array_equal(got, want)
    assert np.signbit(got[128]) and paged.MAGNITUDES[-1] == 448.0


def test_encoding_is_to_nearest_ties_to_even():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(20000, generator=g) * torch.exp2(torch.randint(-12, 9, (20000,), generator=g).float())
    x = torch.cat([x.clamp(-448, 448), torch.tensor([0.0, -0.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11, 448.0])])
    want = x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(paged.encode(x.double().numpy()), want)
    np.testing.assert_array_equal(paged.encode([1e9, -1e9, math.nan, math.inf, -math.inf]), [126, 254, 127, 127, 127])


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_exponent_is_the_least_that_holds_the_largest(kind):
    lo, hi = paged.RANGE[kind]
    for top in [1e-30, 0.1, 1.75, 1.7578125, 448.0, 450.0, 448 * 2.0 ** -7, 5e4]:
        e = paged.exponent([0.0, -top, math.nan, math.inf], lo, hi)
        assert lo <= e <= hi and (top <= 448 * 2.0 ** e or e == hi) and (e == lo or top > 448 * 2.0 ** (e - 1))
    assert paged.exponent([0.0, math.nan], lo, hi) == lo


@pytest.mark.parametrize("kind,dtype", [("bf16", torch.bfloat16), ("f16", torch.float16)])
def test_every_element_is_a_number_of_the_dtype(kind, dtype):
    finite = paged.decode(np.arange(127))
    for e in paged.RANGE[kind]:
        x = torch.from_numpy(np.ldexp(finite, e))
        assert torch.equal(x.to(dtype).double(), x) and torch.isfinite(x.to(dtype)).all()


def test_append_in_pieces():
    """A page filled in two goes: the first numbers within a step of what one go gives,
    the rest as one go gives them; an outlier takes the page's exponent up."""
    g = np.random.default_rng(1)
    x = g.standard_normal((16, 1, 64))
    x[9] *= 64
    one, two = np.zeros((2, 1, 16, 64), np.uint8), np.zeros((2, 1, 16, 64), np.uint8)
    e1, e2 = np.zeros((2, 1), np.int8), np.zeros((2, 1), np.int8)
    paged.append(one, e1, x, 0, [1], 16, -110, 119)
    paged.append(two, e2, x[:5], 0, [1], 16, -110, 119)
    first = int(e2[1, 0])
    paged.append(two, e2, x[5:], 5, [1], 16, -110, 119)
    assert e1[1, 0] == e2[1, 0] > first and not one[0].any()
    a, b = paged.values(one, e1)[1, 0], paged.values(two, e2)[1, 0]
    np.testing.assert_array_equal(a[5:], b[5:])
    step = np.maximum(np.abs(x[:5, 0]) * 2.0 ** -3, math.ldexp(2.0 ** -9, int(e1[1, 0])))
    assert (np.abs(a[:5] - b[:5]) <= step).all()
    assert (np.abs(a - x[:, 0]) <= np.maximum(np.abs(x[:, 0]) * 2.0 ** -4, math.ldexp(2.0 ** -10, int(e1[1, 0])))).all()


def test_fork_worked_example():
    # pages of 16; rows: 20 positions on pages 3, 5; 32 on pages 0, 3 (3 shared)
    refs = [1, 0, 0, 2, 0, 1, 0]
    table = [[3, 5, -9], [0, 3, -9]]
    refs2, out, copies, short = paged.fork(refs, table, [20, 32], [0, 0, 1, -1], [21, 20, 33, 5], 4, 16)
    assert out.tolist() == [[3, 5, -1, -1], [3, 1, -1, -1], [0, 3, 2, -1], [4, -1, -1, -1]]
    assert copies == [(5, 1)] and short == 0
    assert refs2.tolist() == [1, 1, 1, 3, 1, 1, 0]
    # taken back into a page that another row keeps whole: the shorter one gets a copy
    refs2, out, copies, _ = paged.fork([2, 1, 0], [[0, 1]], [32], [0, 0], [20, 32], 2, 16)
    assert out.tolist() == [[0, 2], [0, 1]] and copies == [(1, 2)] and refs2.tolist() == [3, 1, 1]
    # no page left
    _, out, copies, short = paged.fork([1, 1], [[0, 1]], [20], [0], [40], 3, 16)
    assert out.tolist() == [[0, 1, -1]] and short == 1 and not copies


@pytest.mark.parametrize("seed", range(20))
def test_counts_are_the_rows_that_hold_a_page(seed):
    """A pool held by the table alone: afterwards the counts are how often each page
    stands in the new table, open pages stand in one row, and used pages fill the
    beginning after a compaction, each row's in its order."""
    g = np.random.default_rng(seed)
    page, n = 16, 60
    lens = [int(g.integers(0, 70)) for _ in range(5)]
    order = list(g.permutation(n))
    table = np.full((5, 8), -7)
    refs = np.zeros(n, int)
    for b, l in enumerate(lens):
        for j in range((l + 15) // 16):
            table[b, j] = order.pop()
            refs[table[b, j]] += 1
    parents = [int(x) for x in g.integers(-1, 5, 7)]
    after = [int(x) for x in g.integers(0, 90, 7)]
    refs2, out, copies, short = paged.fork(refs, table, lens, parents, after, 8, page)
    assert short == 0
    np.testing.assert_array_equal(np.bincount(out[out >= 0], minlength=n), refs2)
    for i, end in enumerate(after):
        kept = min(end, lens[parents[i]] if parents[i] >= 0 else 0)
        if kept % page:
            assert refs2[out[i, kept // page]] == 1
    refs3, out3, where, moves = paged.compact(refs2, out, after, page)
    u = int((refs2 > 0).sum())
    assert (refs3[:u] > 0).all() and not refs3[u:].any() and sorted(refs3) == sorted(refs2)
    for i, end in enumerate(after):
        m = (end + 15) // 16
        np.testing.assert_array_equal(out3[i, :m], where[out[i, :m]])
    assert all(a >= u > b for a, b in moves)
