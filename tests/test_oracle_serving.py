"""Pins of the serving oracle: rotary against complex multiplication and its
identities, attention against torch's float64 softmax with a mask."""
import numpy as np
import pytest
import torch

from oracle import serving as osv


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotary_is_a_complex_rotation(adjacent):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 2, 16))
    pos = rng.integers(0, 1000, (2, 5))
    f = np.array([1.0, 0.3, 0.05, 0.7, 0.2])
    axis = [0, 1, 1, 0, 1]
    y = osv.rotary(x, pos, f, axis, adjacent, 1.25)
    n = len(f)
    for t in range(5):
        for i in range(n):
            a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
            z = (x[t, :, a] + 1j * x[t, :, b]) * 1.25 * np.exp(1j * pos[axis[i], t] * f[i])
            np.testing.assert_allclose(y[t, :, a], z.real, rtol=0, atol=1e-12)
            np.testing.assert_allclose(y[t, :, b], z.imag, rtol=0, atol=1e-12)
    np.testing.assert_array_equal(y[..., 2 * n:], x[..., 2 * n:])


def test_rotated_scores_depend_on_the_distance():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((1, 1, 8)), rng.standard_normal((1, 1, 8))
    f = [1.0, 0.1, 0.01, 0.001]
    dots = []
    for shift in (0, 17, 400):
        a = osv.rotary(q, [[9 + shift]], f, [0] * 4)
        b = osv.rotary(k, [[2 + shift]], f, [0] * 4)
        dots.append(float((a * b).sum()))
    assert max(dots) - min(dots) < 1e-12


@pytest.mark.parametrize("n,t,window", [(7, 7, 0), (3, 9, 0), (9, 9, 4), (2, 9, 1), (5, 3, 0)])
def test_attend_against_a_masked_softmax(n, t, window):
    rng = np.random.default_rng(2)
    q = rng.standard_normal((n, 6, 8))
    k, v = rng.standard_normal((2, 2, t, 8))
    out, mass, plain, span = osv.attend(q, k, v, 0.4, window)
    qt, kt, vt = (torch.from_numpy(a) for a in (q, k, v))
    x = 0.4 * torch.einsum("nhd,htd->hnt", qt, kt.repeat_interleave(3, 0))
    back = torch.arange(t - n, t)[:, None] - torch.arange(t)
    x = x.masked_fill((back < 0) | (back >= (window or t + n)), -torch.inf)
    ref = torch.nan_to_num(torch.einsum("hnt,htd->nhd", torch.softmax(x, -1), vt.repeat_interleave(3, 0)))
    np.testing.assert_allclose(out, ref.numpy(), rtol=1e-12, atol=1e-13)
    assert (mass >= np.abs(out) - 1e-12).all() and (plain >= mass - 1e-12).all() and (span >= 0).all()


def test_pages_hold_positions_in_table_order():
    pool = np.arange(4 * 1 * 2 * 1).reshape(4, 1, 2, 1)
    got = osv.from_pages(pool, [3, 0, 2], 5, 2)[0, :, 0]
    assert got.tolist() == [6, 7, 0, 1, 4]
    assert [osv.place(t, [3, 0, 2], 2) for t in (0, 3, 4)] == [(3, 0), (0, 1), (2, 0)]
