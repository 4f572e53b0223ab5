"""Serving operators on the GPU against the float64 oracle: rotary positions,
the paged cache's append and attention, attention over whole prompts, and a run
of them together.  Every tolerance is oracle.serving.attend_bound's (or, for
the rotary, the bound beside it), derived from the roundings each path makes."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import serving as osv

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
PI = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
# half the last step below the type's normal range, relative to a row's largest weight
SMALL = {BF16: 0.0, F16: 2.0 ** -25}


def f64(t):
    return t.detach().double().cpu().numpy()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(news):
    return ints(np.concatenate([[0], np.cumsum(news)]).tolist())


def randn(g, shape, dtype=F32):
    return torch.randn(shape, generator=g).to(dtype).cuda()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def close(got, ref, tol, what=""):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape
    assert np.isfinite(got).all(), f"{what}: non-finite output"
    over = np.abs(got - ref) - tol
    assert (over <= 0).all(), f"{what}: {np.abs(got - ref).max():.3e} off, {over.max():.3e} over at {np.unravel_index(over.argmax(), over.shape)}"


# -- rotary ------------------------------------------------------------------------
def rotary_bound(x, ref, inv_freq, pos, dtype, factor, adjacent, n):
    """Rounded once (u); before it each product and sum in binary32 on cos and
    sin within 2^-22 (their own 2 ulp, the turn's 2^-25 as a float, 2^-32 of a
    turn cut off), and the angle's own share of the position times half a step of
    the double that holds the frequency."""
    mag = np.abs(np.asarray(x)).copy()
    a = np.arange(n) * (2 if adjacent else 1)
    b = a + (1 if adjacent else n)
    both = mag[..., a] + mag[..., b]
    far = np.abs(np.asarray(pos, np.float64)).max(0)[:, None, None] * np.max(np.abs(inv_freq)) * 2.0 ** -51
    e = (2.0 ** -21 + far) * both * abs(factor)
    extra = np.zeros_like(mag)
    extra[..., a], extra[..., b] = e, e
    return U[dtype] * np.abs(ref) + extra * (1 + U[dtype]) + (2.0 ** -25 if dtype == F16 else 0.0)


def rotary_case(dtype, head_dim, rotary_dim, axes, adjacent, n_tokens, hq, hk, pos_hi, seed=0, factor=1.0, stride="fused",
                inplace=False):
    from paper_2609_37988_gb300.serving import Rotary
    g = gen(seed)
    n = rotary_dim // 2
    axis = [int(a) for a in torch.randint(0, axes, (n,), generator=g)]
    axis[-1] = axes - 1
    rot = Rotary(head_dim=head_dim, rotary_dim=rotary_dim, base=10000.0, axes=axis, adjacent=adjacent, factor=factor)
    inv_freq = [10000.0 ** (-2.0 * i / rotary_dim) for i in range(n)]
    pos = torch.randint(-pos_hi // 8, pos_hi, (axes, n_tokens), generator=g, dtype=torch.int32)
    extra = {"fused": 1, "odd": 0}[stride]
    if stride == "odd":  # rows that start on no 16-byte boundary
        flat = randn(g, (n_tokens * (hq + hk) * (head_dim + 1) + 1,), dtype)[1:]
        qkv = flat.view(n_tokens, hq + hk, head_dim + 1)[..., :head_dim]
    else:
        qkv = randn(g, (n_tokens, hq + hk + extra, head_dim), dtype)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
    x = f64(qkv)
    out = (q, k) if inplace else None
    oq, ok = rot.apply(q if hq else None, k if hk else None, pos.cuda(), out=out if hq and hk else None)
    for got, lo, h in ((oq, 0, hq), (ok, hq, hk)):
        if not h:
            assert got is None
            continue
        xs = x[:, lo:lo + h]
        ref = osv.rotary(xs, pos.numpy(), inv_freq, axis, adjacent, factor)
        close(got, ref, rotary_bound(xs, ref, inv_freq, pos.numpy(), dtype, factor, adjacent, n))
    if inplace and extra:  # the value head beside them is as it was
        np.testing.assert_array_equal(f64(qkv)[:, hq + hk:], x[:, hq + hk:])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("head_dim,rotary_dim,axes", [(128, 128, 1), (128, 128, 3), (64, 64, 2), (128, 64, 3), (256, 256, 1),
                                                      (80, 80, 3), (96, 24, 2), (2, 2, 1), (64, 6, 8)])
def test_rotary(dtype, adjacent, head_dim, rotary_dim, axes):
    rotary_case(dtype, head_dim, rotary_dim, min(axes, rotary_dim // 2), adjacent, 7, 5, 2, 4096)


@pytest.mark.parametrize("stride,inplace", [("fused", True), ("odd", False), ("odd", True)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rotary_strides_and_in_place(dtype, stride, inplace):
    rotary_case(dtype, 128, 128, 3, False, 9, 4, 2, 100000, stride=stride, inplace=inplace, factor=1.1)
    rotary_case(dtype, 64, 32, 1, True, 9, 4, 2, 100000, stride=stride, inplace=inplace)


@pytest.mark.parametrize("tokens,hq,hk", [(1, 28, 4), (1, 1, 0), (3, 0, 2), (4099, 2, 1), (5, 64, 8)])
def test_rotary_sizes_and_far_positions(tokens, hq, hk):
    rotary_case(F32, 64, 64, 2, False, tokens, hq, hk, 2 ** 30, seed=3)
    rotary_case(BF16, 128, 128, 1, False, tokens, hq, hk, 2 ** 24, seed=4)


def test_rotary_empty():
    from paper_2609_37988_gb300.serving import Rotary
    rot = Rotary(head_dim=64)
    q, k = rot.apply(torch.empty((0, 4, 64), device="cuda"), None, ints([]).view(1, 0))
    assert q.shape == (0, 4, 64) and k is None


# -- batches over pages --------------------------------------------------------------
class Batch:
    """A batch over pages: pools full of NaN, sequences' pages in random order,
    the table's unused entries far outside the pool."""

    def __init__(self, news, lens, hq, hkv, d, dtype, page, seed=0, spare=3, slack=1, rows_behind=0):
        from paper_2609_37988_gb300.serving import PagedCache
        g = gen(seed)
        self.news, self.lens, self.page, self.dtype = news, lens, page, dtype
        self.hq, self.hkv, self.d = hq, hkv, d
        per = [(max(l, 0) + page - 1) // page for l in lens]
        n_pages = sum(per) + spare
        order = torch.randperm(n_pages, generator=g).tolist()
        width = max(per + [0]) + slack
        self.table = np.full((len(lens), width), 2 ** 30, np.int64)
        for b, m in enumerate(per):
            self.table[b, :m] = [order.pop() for _ in range(m)]
        pools = [torch.full((n_pages, hkv, page, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
        self.cache = PagedCache(n_q_heads=hq, k_pages=pools[:1], v_pages=pools[1:])
        self.cu, self.lengths, self.table_d = offsets(news), ints(lens), ints(self.table.tolist())
        # every position's keys and values, the new tokens' too
        self.k = [torch.randn((max(l, 0), hkv, d), generator=g).to(dtype) for l in lens]
        self.v = [torch.randn((max(l, 0), hkv, d), generator=g).to(dtype) for l in lens]
        self.n = sum(news) + rows_behind
        self.q = torch.randn((self.n, hq, d), generator=g).to(dtype)

    def fill(self):
        """All positions through the append, as if all were new."""
        ls = [max(l, 0) for l in self.lens]
        if sum(ls):
            k, v = torch.cat(self.k).cuda(), torch.cat(self.v).cuda()
            self.cache.append(0, k, v, offsets(ls), ints(ls), self.table_d)
        return self

    def expected(self, scale, window, t_max=None):
        out, tol, at = [], [], 0
        for b, (n, l) in enumerate(zip(self.news, self.lens)):
            k, v = (np.transpose(f64(x[b]), (1, 0, 2)) for x in (self.k, self.v))
            if l < n:  # queries before position 0
                k, v = (np.zeros((self.hkv, max(l, 0), self.d)) if not l > 0 else x for x in (k, v))
            r = osv.attend(f64(self.q[at:at + n]), k, v, scale, window)
            if l < 0:
                r = tuple(np.zeros_like(x) for x in r)
            out.append(r[0])
            tol.append(osv.attend_bound(*r, self.d, max(l, 1), U[self.dtype], SMALL[self.dtype]))
            at += n
        return np.concatenate(out), np.concatenate(tol)

    def attend(self, scale, window=0, max_new=None, q=None, **kw):
        return self.cache.attend(0, self.q.cuda() if q is None else q, self.cu, self.lengths, self.table_d, scale,
                                 window=window, max_new=max(self.news + [1]) if max_new is None else max_new, **kw)

    def check(self, window=0, max_new=None):
        scale = 1.0 / math.sqrt(self.d)
        got = self.attend(scale, window, max_new)
        ref, tol = self.expected(scale, window)
        close(got[: sum(self.news)], ref, tol, f"window {window}, max_new {max_new}")
        assert self.cache.device_error() == 0
        return got


HEADS = [(40, 8, 128), (28, 4, 128), (8, 2, 64), (4, 4, 64), (16, 1, 128), (6, 2, 128), (48, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype,page", [(BF16, 16), (F16, 32), (BF16, 64), (F16, 128)])
def test_single_tokens(hq, hkv, d, dtype, page):
    b = Batch([1] * 7, [1, 2, 63, 64, 65, 300, 17], hq, hkv, d, dtype, page).fill()
    for window in (0, 1, 50):
        b.check(window)


@pytest.mark.parametrize("news,lens", [([5, 1, 3, 0, 2], [5, 1, 130, 77, 66]), ([9, 4], [700, 4]), ([1], [2100]), ([3, 1], [1, 0]),
                                       ([2, 0, 0, 6], [513, 0, 9, 64])])
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(40, 8, 128, BF16, 16), (28, 4, 128, F16, 64), (8, 2, 64, BF16, 128)])
def test_few_tokens(news, lens, hq, hkv, d, dtype, page):
    b = Batch(news, lens, hq, hkv, d, dtype, page, seed=5).fill()
    for window in (0, 1, 7, 100):
        b.check(window)
    b.check(0, max_new=sum(news))


CHUNKS = [([70, 33], [70, 500]), ([129, 1, 64, 0, 127], [129, 1, 200, 5, 383]), ([260], [260]), ([31, 300], [1000, 301]),
          ([50, 50], [20, 50])]


@pytest.mark.parametrize("news,lens", CHUNKS)
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(10, 2, 128, BF16, 16), (7, 1, 128, F16, 32), (8, 2, 64, BF16, 64), (3, 3, 64, F16, 16),
                                                 (8, 1, 128, BF16, 128)])
def test_chunks(news, lens, hq, hkv, d, dtype, page):
    b = Batch(news, lens, hq, hkv, d, dtype, page, seed=6).fill()
    for window in (0, 40, 129):
        b.check(window)


@pytest.mark.parametrize("news,lens", [([1, 1], [3000, 77]), ([4, 2], [1000, 130]), ([40, 130], [1000, 700]), ([700], [1500])])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_pages_that_the_window_has_left_need_no_entry(news, lens, page):
    b = Batch(news, lens, 8, 2, 128, BF16, page, seed=31).fill()
    for window in (1, 33, 100, 300):
        stale = b.table.copy()
        for s, (n, m) in enumerate(zip(news, lens)):
            stale[s, :max(0, m - n - window + 1) // page] = -1 if s else 2 ** 30
        b.table_d = ints(stale.tolist())
        b.check(window)


@pytest.mark.parametrize("hq,hkv,d", [(64, 1, 128), (128, 2, 64), (33, 1, 128), (51, 3, 64), (65, 65, 64)])
def test_head_groups_of_every_width(hq, hkv, d):
    """The widest group, groups that fill no tile, many heads of their own; single
    tokens of wide groups go with the chunks."""
    b = Batch([1, 1, 1], [70, 1, 300], hq, hkv, d, BF16, 16, seed=41).fill()
    b.check()
    b = Batch([9, 0, 66], [9, 5, 200], hq, hkv, d, F16, 32, seed=42).fill()
    for window in (0, 50):
        b.check(window)
    prompt_case([1, 77, 140], hq, hkv, d, BF16, windows=(0, 33), seed=43)


RUNS = [([9], [3000]), ([300, 7], [2500, 2100]), ([24, 1, 0, 33], [4000, 10, 70, 1500]), ([600], [2600])]


@pytest.mark.parametrize("news,lens", RUNS)
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(10, 2, 128, BF16, 16), (7, 1, 128, F16, 64), (8, 2, 64, BF16, 128)])
def test_chunks_over_long_contexts(news, lens, hq, hkv, d, dtype, page):
    """Few jobs of many tiles: cut into pieces and joined, in either form of the join."""
    b = Batch(news, lens, hq, hkv, d, dtype, page, seed=51).fill()
    for window in (0, 1300):
        b.check(window)
    first = b.attend(0.1)
    for _ in range(3):
        assert torch.equal(b.attend(0.1)[: sum(news)], first[: sum(news)])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_not_finite_in_pieces_of_jobs(bad):
    news, lens = [80, 150], [2000, 1900]
    b = Batch(news, lens, 10, 2, 128, BF16, 16, seed=52)
    for s, t, ch in [(0, 1999, 3), (1, 1898, 77), (1, 1820, 5), (0, 1950, 127)]:
        b.v[s][t, 1, ch] = bad
    b.k[1][1899, 0, 9] = float("nan")
    b.fill()
    for window in (0, 1200):
        scale = 1.0 / math.sqrt(128)
        got = f64(b.attend(scale, window)[: sum(news)])
        ref, tol = b.expected(scale, window)
        fine = np.isfinite(ref)
        assert (np.isfinite(got) == fine).all()
        assert (np.abs(got[fine] - ref[fine]) <= tol[fine]).all()


def test_chunks_over_long_contexts_captured():
    """A graph of calls whose jobs are cut, replayed as the lengths grow."""
    b = Batch([40, 20], [3000, 2200], 10, 2, 128, BF16, 16, seed=53).fill()
    lens = [2000, 2200]
    b.lengths.copy_(ints(lens))
    q, scale = b.q.cuda(), 1.0 / math.sqrt(128)
    out = torch.empty_like(q)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        for _ in range(2):
            b.attend(scale, q=q, out=out)
    full_k, full_v = b.k, b.v
    for lens in ([2000, 2200], [3000, 100], [60, 2200]):
        b.lengths.copy_(ints(lens))
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        b.k, b.v, b.lens = [x[:m] for x, m in zip(full_k, lens)], [x[:m] for x, m in zip(full_v, lens)], lens
        ref, tol = b.expected(scale, 0)
        close(out, ref, tol, f"lengths {lens}")
    assert b.cache.device_error() == 0


def test_rows_in_no_sequence_stay():
    b = Batch([3, 2], [70, 9], 8, 2, 64, BF16, 16, rows_behind=4).fill()
    out = torch.full((b.n, 8, 64), 7.0, dtype=BF16, device="cuda")
    b.attend(0.125, out=out)
    assert (out[5:] == 7.0).all() and not (out[:5] == 7.0).all()
    out2 = torch.full((b.n, 8, 64), 7.0, dtype=BF16, device="cuda")
    b.attend(0.125, out=out2, max_new=b.n)
    assert (out2[5:] == 7.0).all() and not (out2[:5] == 7.0).all()


@pytest.mark.parametrize("news", [[1, 1], [3, 2], [80, 150]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(news, bad):
    """In keys and values, at a position of the last tile and of an earlier one."""
    lens = [200, 190]
    b = Batch(news, lens, 10, 2, 128, BF16, 16, seed=8)
    places = [(0, lens[0] - 1, 3), (1, lens[1] - 2, 77), (1, lens[1] - news[1] // 2 - 1, 5)]
    for s, t, ch in places:
        b.v[s][t, 1, ch] = bad
    b.k[1][lens[1] - 1, 0, 9] = float("nan")
    b.fill()
    for window in (0, 60):
        scale = 1.0 / math.sqrt(128)
        got = f64(b.attend(scale, window)[: sum(news)])
        ref, tol = b.expected(scale, window)
        fine = np.isfinite(ref)
        assert (np.isfinite(got) == fine).all()
        assert (np.abs(got - ref)[fine] <= tol[fine]).all()


def test_an_infinite_score_is_not_a_number():
    b = Batch([1], [70], 4, 2, 64, BF16, 16, seed=9)
    b.k[0][33, 0, :] = 3e38
    b.q[0, 0, :] = 3e38
    b.fill()
    got = f64(b.attend(0.125))
    assert np.isnan(got[0, 0]).all() and np.isfinite(got[0, 2:]).all()


def test_large_scores_and_equal_rows():
    """Scores far apart (one key takes all), far below zero, and all equal."""
    b = Batch([2, 90], [150, 300], 10, 2, 128, F16, 16, seed=10)
    for s in range(2):
        b.k[s] *= 8
    b.q *= 4
    b.k[1][:] = b.k[1][:1]
    b.fill().check()
    b.check(33)


def test_pages_shared_between_sequences():
    b = Batch([1, 1, 1], [100, 100, 40], 8, 2, 64, BF16, 16, seed=11)
    b.table[1, :5] = b.table[0, :5]
    b.table_d = ints(b.table.tolist())
    b.k[1][:80], b.v[1][:80] = b.k[0][:80], b.v[0][:80]
    b.fill().check()


def test_strided_queries_and_repeated_calls_agree_to_the_bit():
    b = Batch([4, 1, 100], [3000, 1000, 700], 28, 4, 128, BF16, 32, seed=12).fill()
    wide = torch.zeros((b.n, 40, 128), dtype=BF16, device="cuda")
    wide[:, 5:33] = b.q.cuda()
    a = b.attend(0.088, q=wide[:, 5:33])
    for max_new in (None, b.n):
        first = b.attend(0.088, max_new=max_new)
        for _ in range(5):
            assert torch.equal(first, b.attend(0.088, max_new=max_new))
    assert torch.equal(a, b.attend(0.088))
    perm = b.q.cuda().permute(1, 0, 2).contiguous().permute(1, 0, 2)  # heads outermost
    assert torch.equal(a, b.attend(0.088, q=perm))


def test_device_errors_and_recovery():
    b = Batch([1, 2], [80, 90], 8, 2, 64, BF16, 16, seed=13, slack=0).fill()
    keep = b.attend(0.125)
    bad = b.table_d.clone()
    bad[0, 2] = 10 ** 6
    b.cache.attend(0, b.q.cuda(), b.cu, b.lengths, bad, 0.125, max_new=2)
    assert b.cache.device_error() == 32
    bad[0, 2] = -5
    b.cache.attend(0, b.q.cuda(), b.cu, b.lengths, bad, 0.125)
    assert b.cache.device_error() == 32
    # more new tokens than said; more positions than the table holds
    b.attend(0.125, max_new=1)
    assert b.cache.device_error() == 4
    b.cache.attend(0, b.q.cuda(), b.cu, ints([80, 10 ** 6]), b.table_d, 0.125, max_new=2)
    assert b.cache.device_error() == 4
    k = torch.zeros((3, 2, 64), dtype=BF16, device="cuda")
    b.cache.append(0, k, k, b.cu, ints([80, 10 ** 6]), b.table_d)
    assert b.cache.device_error() == 2
    b.cache.append(0, k, k, b.cu, ints([49, 90]), torch.full_like(b.table_d, 10 ** 6))
    assert b.cache.device_error() == 32
    b.fill()
    assert torch.equal(keep, b.attend(0.125)) and b.cache.device_error() == 0


def test_lengths_of_sequences_without_new_tokens_do_not_matter():
    b = Batch([1, 0, 2], [70, 40, 90], 8, 2, 64, BF16, 16, seed=31).fill()
    keep = b.attend(0.125)
    for other in (10 ** 9, -5):
        got = b.cache.attend(0, b.q.cuda(), b.cu, ints([70, other, 90]), b.table_d, 0.125, max_new=2)
        assert torch.equal(keep, got) and b.cache.device_error() == 0
        got = b.cache.attend(0, b.q.cuda(), b.cu, ints([70, other, 90]), b.table_d, 0.125, max_new=40)
        assert b.cache.device_error() == 0


@pytest.mark.parametrize("news", [[1, 2], [40, 70]])
def test_pools_past_two_to_the_31_elements(news):
    """Pages at both ends of pools of 2^31 + elements."""
    from paper_2609_37988_gb300.serving import PagedCache
    hq, hkv, d, page = 8, 8, 128, 128
    n_pages = 2 ** 31 // (hkv * page * d) + 4
    cache = PagedCache(n_q_heads=hq, n_kv_heads=hkv, n_layers=1, head_dim=d, n_pages=n_pages, page_size=page, dtype=BF16)
    lens = [300, 200]
    table = np.array([[n_pages - 1, 0, n_pages - 3], [n_pages - 2, 1, 0]])
    g = gen(32)
    k, v = [torch.randn((l, hkv, d), generator=g).to(BF16) for l in lens], [torch.randn((l, hkv, d), generator=g).to(BF16) for l in lens]
    q = torch.randn((sum(news), hq, d), generator=g).to(BF16)
    cache.append(0, torch.cat(k).cuda(), torch.cat(v).cuda(), offsets(lens), ints(lens), ints(table.tolist()))
    got = cache.attend(0, q.cuda(), offsets(news), ints(lens), ints(table.tolist()), 0.088, max_new=max(news))
    at = 0
    for b, n in enumerate(news):
        r = osv.attend(f64(q[at:at + n]), *(np.transpose(f64(x[b]), (1, 0, 2)) for x in (k, v)), 0.088)
        close(got[at:at + n], r[0], osv.attend_bound(*r, d, lens[b], U[BF16], 0.0))
        at += n
    assert cache.device_error() == 0


def test_two_caches_over_the_same_pools_at_once():
    """Workspaces are a cache object's own: two of them run side by side."""
    from paper_2609_37988_gb300.serving import PagedCache
    a = Batch([1, 2, 1], [900, 300, 5], 10, 2, 128, BF16, 16, seed=33).fill()
    b = Batch([30, 80], [700, 900], 10, 2, 128, BF16, 16, seed=34).fill()
    twin = PagedCache(n_q_heads=10, k_pages=b.cache.k_pages, v_pages=b.cache.v_pages)
    keep_a, keep_b = a.attend(0.088), b.attend(0.088)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    qa, qb = a.q.cuda(), b.q.cuda()
    torch.cuda.synchronize()
    outs = []
    for _ in range(10):
        outs.append((keep_a, a.attend(0.088, q=qa, stream=streams[0])))
        outs.append((keep_b, b.attend(0.088, q=qb, stream=streams[1])))
        outs.append((keep_b, twin.attend(0, qb, b.cu, b.lengths, b.table_d, 0.088, max_new=80, stream=streams[2])))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in outs)


def test_empty_batches():
    b = Batch([0, 0], [0, 40], 8, 2, 64, BF16, 16).fill()
    assert b.attend(0.125).shape == (0, 8, 64)
    q = torch.full((3, 8, 64), 5.0, dtype=BF16, device="cuda")
    out = b.attend(0.125, q=q, out=q.clone(), max_new=3)
    assert (out == 5.0).all()
    none = torch.zeros((0,), dtype=torch.int32, device="cuda")
    b.cache.attend(0, q, ints([0]), none, torch.zeros((0, 3), dtype=torch.int32, device="cuda"), 0.125)
    assert b.cache.device_error() == 0


@pytest.mark.parametrize("news,lens", [([1, 1, 1], [500, 2, 77]), ([64, 200], [64, 900])])
def test_captured_and_replayed_on_another_stream(news, lens):
    b = Batch(news, lens, 10, 2, 128, BF16, 16, seed=14).fill()
    scale = 1.0 / math.sqrt(128)
    keep = b.attend(scale)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q, out = b.q.cuda(), torch.empty_like(keep)
    b.attend(scale, q=q, out=out, stream=side)
    side.synchronize()
    assert torch.equal(keep, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.attend(scale, q=q, out=out)
        b.attend(scale, q=q, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(keep, out)
    # the lengths are read when the graph runs
    b.lengths.copy_(ints([max(n, l - 1) for n, l in zip(news, lens)]))
    graph.replay()
    torch.cuda.synchronize()
    b.lens = [max(n, l - 1) for n, l in zip(news, lens)]
    b.k = [x[:l] for x, l in zip(b.k, b.lens)]
    b.v = [x[:l] for x, l in zip(b.v, b.lens)]
    ref, tol = b.expected(scale, 0)
    close(out, ref, tol)


# -- append ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,page,hq,hkv,d", [(BF16, 16, 10, 2, 128), (F16, 64, 8, 2, 64), (BF16, 128, 3, 3, 64), (F16, 32, 28, 4, 128)])
@pytest.mark.parametrize("mode", ["plain", "rotary", "own positions", "odd strides"])
def test_append(dtype, page, hq, hkv, d, mode):
    from paper_2609_37988_gb300.serving import Rotary
    news, lens = [3, 0, 1, 40, 6], [3, 5, 129, 200, 4]
    b = Batch(news, lens, hq, hkv, d, dtype, page, seed=15, rows_behind=2)
    n = b.n
    g = gen(16)
    if mode == "odd strides":
        flat = randn(g, (n * (hq + 2 * hkv) * (d + 1) + 1,), dtype)[1:]
        qkv = flat.view(n, hq + 2 * hkv, d + 1)[..., :d]
    else:
        qkv = randn(g, (n, hq + 2 * hkv, d), dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    sections = [d // 2] if mode == "own positions" else [d // 8, d // 8, d // 4]
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    rot = Rotary(head_dim=d, base=1e6, sections=sections)
    inv_freq = [1e6 ** (-2.0 * i / d) for i in range(d // 2)]
    pos = torch.randint(0, 50000, (3, n), generator=g, dtype=torch.int32)
    own = np.concatenate([np.arange(l - m, l) for m, l in zip(news, lens)] + [np.zeros(2)])[None]
    before = [f64(t) for t in (b.cache.k_pages[0], b.cache.v_pages[0])]
    kw = {} if mode == "plain" else dict(rotary=rot, positions=None if mode == "own positions" else pos.cuda(), q=q)
    q_out = torch.full((n, hq, d), 7.0, dtype=dtype, device="cuda")
    got = b.cache.append(0, k, v, b.cu, b.lengths, b.table_d, q_out=q_out if kw else None, **kw)
    assert b.cache.device_error() == 0
    rk, tol_k = f64(k), np.zeros((n, hkv, d))
    if kw:
        p = own if mode == "own positions" else pos.numpy()
        rk = osv.rotary(f64(k), p, inv_freq, axis)
        tol_k = rotary_bound(f64(k), rk, inv_freq, p, dtype, 1.0, False, d // 2)
        ref = osv.rotary(f64(q), p, inv_freq, axis)
        m = sum(news)
        close(got[:m], ref[:m], rotary_bound(f64(q), ref, inv_freq, p, dtype, 1.0, False, d // 2)[:m])
        assert (got[m:] == 7.0).all()
    else:
        assert got is None
    after = [f64(t) for t in (b.cache.k_pages[0], b.cache.v_pages[0])]
    at = 0
    for s, (m, l) in enumerate(zip(news, lens)):
        for j in range(m):
            t = l - m + j
            if t >= 0:
                pg, sl = osv.place(t, b.table[s], page)
                close(after[0][pg, :, sl], rk[at + j], tol_k[at + j])
                np.testing.assert_array_equal(after[1][pg, :, sl], f64(v)[at + j])
                for x in (0, 1):
                    before[x][pg, :, sl] = after[x][pg, :, sl]
        at += m
    for x in (0, 1):  # nothing else was written
        np.testing.assert_array_equal(before[x], after[x])


def test_append_rotates_queries_in_place():
    from paper_2609_37988_gb300.serving import Rotary
    b = Batch([5, 4000], [5, 4000], 4, 2, 64, BF16, 16, seed=17)
    rot = Rotary(head_dim=64)
    k, v, q = (randn(gen(18), (4005, h, 64), BF16) for h in (2, 2, 4))
    a = b.cache.append(0, k, v, b.cu, b.lengths, b.table_d, rotary=rot, q=q)
    pos = torch.cat([torch.arange(5), torch.arange(4000)]).to(torch.int32).cuda()
    c, d = rot.apply(q, k, pos)
    assert torch.equal(a, c)
    same = b.cache.append(0, k, v, b.cu, b.lengths, b.table_d, rotary=rot, q=q, q_out=q)
    assert same is q and torch.equal(a, q)
    b2 = Batch([5, 4000], [5, 4000], 4, 2, 64, BF16, 16, seed=17)
    b2.cache.append(0, d, v, b2.cu, b2.lengths, b2.table_d)
    for x, y in ((b.cache.k_pages[0], b2.cache.k_pages[0]), (b.cache.v_pages[0], b2.cache.v_pages[0])):
        assert torch.equal(x.nan_to_num(3.0), y.nan_to_num(3.0))


# -- prompts -----------------------------------------------------------------------------
def prompt_case(lens, hq, hkv, d, dtype, windows=(0,), seed=0, behind=0, first=0, mul=1.0, strided=False):
    from paper_2609_37988_gb300.serving import prompt_attention
    g = gen(seed)
    n = first + sum(lens) + behind
    if strided:
        qkv = randn(g, (n, hq + 2 * hkv + 1, d), dtype)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:hq + 2 * hkv]
    else:
        q, k, v = (randn(g, (n, h, d), F32) for h in (hq, hkv, hkv))
        q, k, v = (q * mul).to(dtype), (k * mul).to(dtype), v.to(dtype)
    cu = ints((first + np.concatenate([[0], np.cumsum(lens)])).tolist())
    error = ints([0])
    scale = 1.0 / math.sqrt(d)
    for window in windows:
        out = torch.full((n, hq, d), 7.0, dtype=dtype, device="cuda")
        got = prompt_attention(q, k, v, cu, scale, window=window, out=out, error=error)
        at = first
        for m in lens:
            r = osv.attend(f64(q[at:at + m]), *(np.transpose(f64(x[at:at + m]), (1, 0, 2)) for x in (k, v)), scale, window)
            close(got[at:at + m], r[0], osv.attend_bound(*r, d, max(m, 1), U[dtype], SMALL[dtype]), f"length {m}, window {window}")
            at += m
        assert (got[:first] == 7.0).all() and (got[at:] == 7.0).all()
        assert int(error) == 0


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_prompts_of_every_head_layout(hq, hkv, d, dtype):
    prompt_case([1, 0, 37, 2, 140], hq, hkv, d, dtype, windows=(0, 19), behind=3)


@pytest.mark.parametrize("lens", [[1], [2], [25, 26], [51, 52, 53], [127, 128, 129], [255, 256, 257], [385], [0, 0, 64, 0]])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(5, 1, 128, BF16), (2, 1, 64, F16), (1, 1, 128, F16)])
def test_prompt_lengths(lens, hq, hkv, d, dtype):
    prompt_case(lens, hq, hkv, d, dtype, windows=(0, 1, 64, 100, 1000), seed=21, first=2)


@pytest.mark.parametrize("mul", [0.05, 4.0])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_prompt_score_ranges(mul, dtype):
    prompt_case([300, 90], 4, 2, 128, dtype, seed=22, mul=mul)


def test_prompt_strides():
    prompt_case([130, 5, 260], 10, 2, 128, BF16, windows=(0, 70), seed=23, strided=True)
    prompt_case([130, 5, 260], 8, 2, 64, F16, seed=24, strided=True)


@pytest.mark.parametrize("count,longest", [(90, 40), (128, 60), (129, 60), (400, 30)])
def test_prompts_many_sequences(count, longest):
    rng = np.random.default_rng(25)
    prompt_case([int(x) for x in rng.integers(0, longest, count)], 4, 2, 64, BF16, seed=25)
    prompt_case([0] * (count - 2) + [300, 1], 2, 1, 128, F16, seed=26)


@pytest.mark.parametrize("count", [33, 130])
@pytest.mark.parametrize("most", [1, 3, 40])
def test_many_sequences_over_pages(count, most):
    rng = np.random.default_rng(27)
    news = [int(x) for x in rng.integers(0, most + 1, count)]
    lens = [int(x) for x in rng.integers(0, 70, count)]
    Batch(news, lens, 10, 2, 64, BF16, 16, seed=28).fill().check(25)


@pytest.mark.parametrize("bad", [float("nan"), float("-inf")])
def test_prompt_values_that_are_not_finite(bad):
    from paper_2609_37988_gb300.serving import prompt_attention
    g = gen(26)
    lens, hq, hkv, d = [300, 170], 5, 1, 128
    q, k, v = (randn(g, (470, h, d), BF16) for h in (hq, hkv, hkv))
    for t, ch in ((120, 0), (299, 64), (303, 127), (469, 3)):
        v[t, 0, ch] = bad
    k[140, 0, 3] = float("nan")
    for window in (0, 90):
        got = f64(prompt_attention(q, k, v, offsets(lens), 0.088, window=window))
        at = 0
        for m in lens:
            r = osv.attend(f64(q[at:at + m]), *(np.transpose(f64(x[at:at + m]), (1, 0, 2)) for x in (k, v)), 0.088, window)
            fine = np.isfinite(r[0])
            x = got[at:at + m]
            assert (np.isfinite(x) == fine).all(), (m, window)
            tol = osv.attend_bound(*r, d, m, U[BF16], 0.0)
            assert (np.abs(x - r[0])[fine] <= tol[fine]).all()
            at += m


def test_prompt_captured_and_repeated():
    from paper_2609_37988_gb300.serving import prompt_attention
    g = gen(27)
    lens = [700, 33, 260]
    q, k, v = (randn(g, (993, h, 128), BF16) for h in (10, 2, 2))
    cu = offsets(lens)
    keep = prompt_attention(q, k, v, cu, 0.088)
    for _ in range(5):
        assert torch.equal(keep, prompt_attention(q, k, v, cu, 0.088))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = prompt_attention(q, k, v, cu, 0.088, stream=side)
    side.synchronize()
    assert torch.equal(keep, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = prompt_attention(q, k, v, cu, 0.088)
        c = prompt_attention(q, k, v, cu, 0.088)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(keep, a) and torch.equal(keep, c)


def test_prompt_offsets_out_of_order_are_clamped():
    from paper_2609_37988_gb300.serving import prompt_attention
    q, k, v = (randn(gen(28), (50, h, 64), BF16) for h in (2, 1, 1))
    out = torch.full((50, 2, 64), 7.0, dtype=BF16, device="cuda")
    prompt_attention(q, k, v, ints([0, 20, 10, 10 ** 6, -3]), 0.125, out=out)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()


# -- together ------------------------------------------------------------------------------
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(10, 2, 128, BF16, 16), (8, 2, 64, F16, 64)])
def test_prompts_then_chunks_then_steps(hq, hkv, d, dtype, page):
    """Prompts attend to themselves and enter the pages, a chunk follows, then
    single tokens: every output against the oracle over all positions so far,
    and the prompt's own attention against the pages' attention of the same."""
    from paper_2609_37988_gb300.serving import PagedCache, Rotary, prompt_attention
    g = gen(30)
    B, stages = 3, [[140, 7, 65], [30, 61, 1], [1, 1, 1], [1, 1, 1]]
    total = [sum(s[b] for s in stages) for b in range(B)]
    rot = Rotary(head_dim=d, base=1e6)
    inv_freq = [1e6 ** (-2.0 * i / d) for i in range(d // 2)]
    per = [(t + page - 1) // page for t in total]
    order = torch.randperm(sum(per), generator=g).tolist()
    table = np.zeros((B, max(per)), np.int64)
    for b in range(B):
        table[b, :per[b]] = [order.pop() for _ in range(per[b])]
    cache = PagedCache(n_layers=2, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, n_pages=sum(per), page_size=page, dtype=dtype)
    scale, held = 1.0 / math.sqrt(d), [0] * B
    seen = [[np.zeros((0, hkv, d))] * 2 for _ in range(B)]
    for i, news in enumerate(stages):
        n = sum(news)
        qkv = randn(g, (n, hq + 2 * hkv, d), dtype)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        held = [h + m for h, m in zip(held, news)]
        cu, lengths, tab = offsets(news), ints(held), ints(table.tolist())
        qr = cache.append(1, k, v, cu, lengths, tab, rotary=rot, q=q)
        pos = ints(np.concatenate([np.arange(h - m, h) for m, h in zip(news, held)]).tolist())
        q2, k2 = rot.apply(q, k, pos)
        assert torch.equal(qr, q2)
        out = cache.attend(1, qr, cu, lengths, tab, scale, max_new=max(news))
        if i == 0:
            own = prompt_attention(q2, k2, v, cu, scale)
        at = 0
        for b, m in enumerate(news):
            rows = slice(at, at + m)
            seen[b] = [np.concatenate([a, f64(x[rows])]) for a, x in zip(seen[b], (k2, v))]
            # the keys as the pages hold them
            pool = f64(cache.k_pages[1])
            np.testing.assert_array_equal(np.transpose(osv.from_pages(pool, table[b], held[b], page), (1, 0, 2)), seen[b][0])
            r = osv.attend(f64(qr[rows]), *(np.transpose(a, (1, 0, 2)) for a in seen[b]), scale)
            tol = osv.attend_bound(*r, d, held[b], U[dtype], SMALL[dtype])
            close(out[rows], r[0], tol, f"stage {i}")
            if i == 0:
                close(own[rows], r[0], tol, "prompt")
            at += m
    assert cache.device_error() == 0


@pytest.mark.parametrize("gap", [12.0, 15.0, 17.5, 20.0])
@pytest.mark.parametrize("d,page,positions", [(128, 16, 4096), (64, 128, 4096), (128, 32, 400)])
def test_f16_weights_far_below_the_largest(gap, d, page, positions):
    """One key `gap` above all the others, its value zero: the result is what the
    others' small weights bring.  They enter the product 2^14 times (few tokens) or
    2^8 times (chunks) as large as the row's largest one is 1, so that half the last
    step below f16's normal range is 2^-39 or 2^-33 of it."""
    b = Batch([1], [positions], 2, 1, d, F16, page, seed=61, rows_behind=20)
    b.q.zero_()
    b.q[..., 0] = 1.0
    b.k[0].zero_()
    b.k[0][positions // 3, 0, 0] = gap
    b.v[0][:] = 1024.0 + 4 * torch.arange(d)
    b.v[0][positions // 3] = 0.0
    b.fill()
    r = osv.attend(f64(b.q[:1]), *(np.transpose(f64(x[0]), (1, 0, 2)) for x in (b.k, b.v)), 1.0)
    for max_new, small in ((1, 2.0 ** -39), (b.n, 2.0 ** -33)):
        got = b.attend(1.0, max_new=max_new)[:1]
        close(got, r[0], osv.attend_bound(*r, d, positions, U[F16], small), f"max_new {max_new}")


def turn_of(f, p):
    """p * f / (2 pi) as a fraction of a turn in [-1/2, 1/2), from f's own binary value."""
    x = Fraction(f) * p / (2 * PI)
    return x - math.floor(x + Fraction(1, 2))


@pytest.mark.parametrize("positive", [True, False])
@pytest.mark.parametrize("freqs", [[1.0, -1.0, 1e-3, -1e-3, 0.75, -0.5, 3.0, 40.0],
                                   [10000.0 ** (-i / 64) for i in range(0, 32, 4)],
                                   [-(1000000.0 ** (-i / 64)) for i in range(3, 35, 4)]])
def test_rotary_angles_at_far_positions(freqs, positive):
    """Angles near whole turns at positions near 2^31, where the angle's 32 bits are
    exact in binary32 and its sine is small: what is left is the 2^-32 of a turn cut
    off, the position times 2^-63 of a turn (the step's own rounding) and 2 ulp of a
    sine below 2^-5 (2^-28)."""
    from paper_2609_37988_gb300.serving import Rotary
    n, tokens = len(freqs), 12
    pos = np.zeros((n, tokens), np.int64)
    for i, f in enumerate(freqs):
        found, p, per = [], 2 ** 31 - 1, Fraction(abs(f)) / (2 * PI)
        while len(found) < tokens:
            p = min(p - 1, math.floor(math.floor(p * per) / per) + 1)  # about a turn back
            for c in (p, p - 1):
                if len(found) < tokens and abs(turn_of(f, c)) < Fraction(1, 300):
                    found.append(c)
            p -= 1
        pos[i] = found
    if not positive:
        pos = -pos
    rot = Rotary(head_dim=2 * n, inv_freq=freqs, axes=list(range(n)))
    x = torch.zeros((tokens, 1, 2 * n), device="cuda")
    x[..., :n] = 1.0
    got = f64(rot.apply(x, None, ints(pos.tolist()))[0])[:, 0]
    tol = 2 * math.pi * (2.0 ** -32 + 2.0 ** 31 * 2.0 ** -63) + 2.0 ** -28
    for i, f in enumerate(freqs):
        for t in range(tokens):
            want = math.sin(2 * math.pi * float(turn_of(f, int(pos[i, t]))))
            assert abs(got[t, n + i] - want) <= tol, (f, int(pos[i, t]), got[t, n + i] - want)


@pytest.mark.parametrize("what", ["prompt", "chunk", "few"])
def test_first_call_of_a_thread(what):
    """Tensor maps of a call's queries are encoded by the driver, which wants a
    current context; a thread that has made no call yet has none."""
    import threading
    from paper_2609_37988_gb300.serving import prompt_attention
    b = Batch([70, 33] if what == "chunk" else [1, 1], [700, 500], 10, 2, 128, BF16, 16, seed=76).fill()
    q, k, v = (randn(gen(77), (200, h, 128), BF16) for h in (10, 2, 2))
    cu, bq = offsets([150, 50]), b.q.cuda()
    out = torch.empty_like(q if what == "prompt" else bq)
    call = {"prompt": lambda: prompt_attention(q, k, v, cu, 0.088, out=out)}.get(what, lambda: b.attend(0.088, q=bq, out=out))
    keep = call().clone()
    out.zero_()
    torch.cuda.synchronize()
    failed = []

    def work():
        try:
            call()
        except Exception as e:
            failed.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not failed and torch.equal(out, keep)


def test_calls_of_several_threads_on_one_stream():
    """An attention that cuts its work is two launches around one list in the
    cache's workspace: threads that share the cache and a stream may call at the
    same time all the same."""
    import threading
    b = Batch([1, 2, 1, 33], [3000, 900, 50, 2000], 10, 2, 128, BF16, 16, seed=62).fill()
    q, scale = b.q.cuda(), 0.088
    # few tokens of three sequences and of one, a chunk, all of them
    calls = []
    for s in ([0, 1, 2], [0], [3], [0, 1, 2, 3]):
        at = np.concatenate([[0], np.cumsum(b.news)])
        rows = torch.cat([torch.arange(at[i], at[i + 1]) for i in s]).cuda()
        calls.append((q[rows].contiguous(), offsets([b.news[i] for i in s]), b.lengths[s].contiguous(),
                      b.table_d[s].contiguous(), max(b.news[i] for i in s)))
    run = lambda c, **kw: b.cache.attend(0, *c[:4], scale, max_new=c[4], **kw)  # noqa: E731
    want = [run(c) for c in calls]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    got, start = [[] for _ in calls], threading.Barrier(len(calls))

    def work(i):
        start.wait()
        for _ in range(100):
            got[i].append(run(calls[i], stream=stream))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    stream.synchronize()
    assert b.cache.device_error(stream) == 0
    for x, w in zip(got, want):
        assert len(x) == 100 and all(torch.equal(y, w) for y in x)


# few tokens in whole units and in runs, chunks in whole jobs and in runs
FORMS = [([1, 2, 1], [300, 2, 77], 0), ([1, 2, 1], [3000, 700, 5], 0), ([200, 70], [400, 500], 0), ([300, 7], [2500, 2100], 0),
         ([24, 1, 0, 33], [4000, 10, 70, 1500], 1000)]


@pytest.mark.parametrize("news,lens,window", FORMS)
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(10, 2, 128, BF16, 16), (8, 2, 64, F16, 64)])
def test_attention_gives_up_and_recovers(news, lens, window, hq, hkv, d, dtype, page):
    """No tile is copied, and every wait for one gives up: the call sets the timeout
    error (and nothing else) and returns; the next one is as before."""
    b = Batch(news, lens, hq, hkv, d, dtype, page, seed=75).fill()
    keep = b.check(window)
    scale, n = 1.0 / math.sqrt(d), sum(news)
    for _ in range(2):
        b.cache.set_give_up(True)
        b.attend(scale, window)
        assert b.cache.device_error() == 8
        b.cache.set_give_up(False)
        assert torch.equal(keep[:n], b.attend(scale, window)[:n]) and b.cache.device_error() == 0


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F16)])
def test_prompts_that_give_up_leave_a_sign(d, dtype):
    """In the caller's word, or in the library's where the caller gives none."""
    from paper_2609_37988_gb300.serving import prompt_attention, prompt_error, prompt_give_up
    q, k, v = (randn(gen(78), (700, h, d), dtype) for h in (10, 2, 2))
    cu, error = offsets([300, 1, 33, 366]), ints([0])
    keep = prompt_attention(q, k, v, cu, 0.088)
    assert prompt_error() == 0
    try:
        prompt_give_up(True)
        prompt_attention(q, k, v, cu, 0.088)
        assert prompt_error() == 8 and prompt_error() == 0
        prompt_attention(q, k, v, cu, 0.088, error=error)
        assert int(error) == 8 and prompt_error(q.device) == 0
    finally:
        prompt_give_up(False)
    error.zero_()
    assert torch.equal(keep, prompt_attention(q, k, v, cu, 0.088)) and prompt_error() == 0
    assert torch.equal(keep, prompt_attention(q, k, v, cu, 0.088, error=error)) and int(error) == 0


def test_prompts_whose_first_call_is_captured():
    """The library's error word is looked up within the capture."""
    import subprocess
    import sys
    program = """
import torch
from paper_2609_37988_gb300.serving import prompt_attention, prompt_error
q, k, v = (torch.randn((200, h, 64), device="cuda").bfloat16() for h in (4, 2, 2))
cu = torch.tensor([0, 150, 200], dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = prompt_attention(q, k, v, cu, 0.125)
graph.replay()
assert prompt_error() == 0 and torch.equal(out, prompt_attention(q, k, v, cu, 0.125))
"""
    subprocess.run([sys.executable, "-c", program], check=True, timeout=120)


def ragged_batch(count, most, longest, seed):
    """News and lengths with empty sequences, short ones and, past the 32nd, long ones."""
    rng = np.random.default_rng(seed)
    news = [int(x) for x in rng.integers(0, most + 1, count)]
    lens = [int(x) for x in rng.integers(0, 80, count)]
    for b in list(rng.integers(0, count, 6)) + [count - 1]:
        news[b], lens[b] = most, int(rng.integers(longest // 2, longest))
    news[5] = news[31] = 0
    return news, lens


@pytest.mark.parametrize("count", [33, 64, 130])
@pytest.mark.parametrize("most", [1, 3])
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(10, 2, 64, BF16, 16), (4, 4, 128, F16, 32)])
def test_few_tokens_of_many_sequences_in_runs(count, most, hq, hkv, d, dtype, page):
    """Over tables of more than 512 positions units are cut into equal runs, whose
    starts are searched 32 sequences at a time."""
    news, lens = ragged_batch(count, most, 900, 63)
    b = Batch(news, lens, hq, hkv, d, dtype, page, seed=63).fill()
    assert b.table.shape[1] * page > 512
    for window in (0, 100):
        first = b.check(window)
        for _ in range(3):
            assert torch.equal(first[: sum(news)], b.attend(1.0 / math.sqrt(d), window)[: sum(news)])


@pytest.mark.parametrize("count", [33, 64, 130])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(5, 1, 128, BF16), (8, 1, 64, F16)])
def test_chunks_of_many_sequences_in_runs(count, hq, hkv, d, dtype):
    """The same for chunks.  One block of tokens a sequence and one KV head are 33 to
    130 jobs of 152 places; behind a table of 2^16 positions the idle ones weigh
    0.14 x 512 tiles and more, and runs are taken."""
    news, lens = ragged_batch(count, 20, 1500, 64)
    page = 16
    b = Batch(news, lens, hq, hkv, d, dtype, page, seed=64, slack=2 ** 16 // page).fill()
    for window in (0, 100):  # (a window bounds the tiles that a place can idle: whole jobs)
        first = b.check(window)
        for _ in range(3):
            assert torch.equal(first[: sum(news)], b.attend(1.0 / math.sqrt(d), window)[: sum(news)])


@pytest.mark.parametrize("tokens", [5003, 9613])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rotary_many_tokens_a_block(tokens, dtype):
    """Narrow rows of many tokens: 8 and 16 tokens of a block."""
    rotary_case(dtype, 64, 64, 3, False, tokens, 8, 2, 4096, seed=65)
    rotary_case(dtype, 64, 32, 1, True, tokens, 3, 1, 4096, seed=66, inplace=True)


@pytest.mark.parametrize("tokens", [5003, 9613])
@pytest.mark.parametrize("own", [True, False])
def test_append_many_tokens_a_block(tokens, own):
    """8 and 16 tokens of a block, sequences that begin and end inside one, a few
    tokens in none."""
    from paper_2609_37988_gb300.serving import Rotary
    news = [3, 0, 1, 40, 2, 700, 5]
    news.append(tokens - sum(news) - 4)
    lens = [n + x for n, x in zip(news, [0, 9, 300, -5, 13, 77, 100, 1])]
    hq, hkv, d, page = 8, 2, 64, 32
    b = Batch(news, lens, hq, hkv, d, BF16, page, seed=67, rows_behind=4)
    assert b.n == tokens
    g = gen(68)
    q, k, v = (randn(g, (tokens, h, d), BF16) for h in (hq, hkv, hkv))
    axis = [0] * (d // 2) if own else [i % 3 for i in range(d // 2)]
    rot = Rotary(head_dim=d, axes=axis)
    inv_freq = [10000.0 ** (-2.0 * i / d) for i in range(d // 2)]
    at = np.concatenate([[0], np.cumsum(news)])
    place = np.concatenate([np.arange(l - n, l) for n, l in zip(news, lens)])
    pos = torch.randint(0, 4096, (3, tokens), generator=g, dtype=torch.int32)
    p = np.concatenate([place, np.zeros(4, np.int64)])[None] if own else pos.numpy()
    q_out = torch.full((tokens, hq, d), 7.0, dtype=BF16, device="cuda")
    b.cache.append(0, k, v, b.cu, b.lengths, b.table_d, rotary=rot, positions=None if own else pos.cuda(), q=q, q_out=q_out)
    assert b.cache.device_error() == 0
    m = sum(news)
    ref = osv.rotary(f64(q), p, inv_freq, axis)
    close(q_out[:m], ref[:m], rotary_bound(f64(q), ref, inv_freq, p, BF16, 1.0, False, d // 2)[:m])
    assert (q_out[m:] == 7.0).all()
    rk = osv.rotary(f64(k), p, inv_freq, axis)
    tol = rotary_bound(f64(k), rk, inv_freq, p, BF16, 1.0, False, d // 2)
    kp, vp = f64(b.cache.k_pages[0]), f64(b.cache.v_pages[0])
    written = np.zeros(kp.shape[:1] + kp.shape[2:3], bool)
    for s in range(len(news)):
        t = place[at[s]:at[s + 1]]
        rows = np.arange(at[s], at[s + 1])[t >= 0]
        t = t[t >= 0]
        pages, slots = b.table[s][t // page], t % page
        close(kp[pages, :, slots], rk[rows], tol[rows])
        np.testing.assert_array_equal(vp[pages, :, slots], f64(v)[rows])
        written[pages, slots] = True
    for pool in (kp, vp):  # nothing else was written
        assert np.isnan(np.transpose(pool, (0, 2, 1, 3))[~written]).all()


def test_lengths_of_sequences_without_new_tokens_do_not_matter_to_chunks():
    b = Batch([40, 0, 25], [70, 40, 90], 8, 2, 64, BF16, 16, seed=69).fill()
    keep = b.check()
    for other in (10 ** 9, -5):
        b.lengths.copy_(ints([70, other, 90]))
        assert torch.equal(keep, b.attend(0.125)) and b.cache.device_error() == 0


def test_prompt_offsets_out_of_order_give_each_sequence_its_own_rows():
    """Offsets 0, 20, 10, 10^6, -3 of 50 tokens are clamped to sequences of tokens
    0 .. 19, none, 10 .. 49 and none; 10 .. 19 belong to two and hold either's rows."""
    from paper_2609_37988_gb300.serving import prompt_attention
    d = 64
    q, k, v = (randn(gen(28), (50, h, d), BF16) for h in (2, 1, 1))
    out = torch.full((50, 2, d), 7.0, dtype=BF16, device="cuda")
    prompt_attention(q, k, v, ints([0, 20, 10, 10 ** 6, -3]), 0.125, out=out)
    for first, last, seen in ((0, 20, slice(0, 10)), (10, 50, slice(10, 40))):
        r = osv.attend(f64(q[first:last]), *(np.transpose(f64(x[first:last]), (1, 0, 2)) for x in (k, v)), 0.125)
        tol = osv.attend_bound(*r, d, last - first, U[BF16], 0.0)
        close(out[first:last][seen], r[0][seen], tol[seen], f"tokens {first} to {last}")


@pytest.mark.parametrize("news,lens", [([1, 1], [65001, 300]), ([2, 3], [64, 65536]), ([33], [65500]), ([1, 17, 0], [40001, 9, 70])])
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(4, 1, 128, BF16, 16), (6, 2, 64, F16, 64)])
def test_contexts_of_65536_positions(news, lens, hq, hkv, d, dtype, page):
    b = Batch(news, lens, hq, hkv, d, dtype, page, seed=71).fill()
    for window in (0, 5000):
        b.check(window)


@pytest.mark.parametrize("news,lens", [([1, 1, 1], [300, 1, 512]), ([1], [512]), ([3, 0, 2], [70, 5, 2]), ([100], [100]), ([600], [600]),
                                       ([64, 1, 30], [64, 400, 31])])
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(10, 2, 128, BF16, 16), (8, 2, 64, F16, 128)])
def test_tables_much_wider_than_the_contexts(news, lens, hq, hkv, d, dtype, page):
    """As a serving program keeps them: a table of 32768 positions, whatever is held.
    Its unused entries lie far outside the pool."""
    b = Batch(news, lens, hq, hkv, d, dtype, page, seed=72, slack=32768 // page).fill()
    for window in (0, 50):
        first = b.check(window)
        assert torch.equal(first, b.attend(1.0 / math.sqrt(d), window))


@pytest.mark.parametrize("news,lens", [([1, 1, 1], [300, 1, 400]), ([1, 2], [3000, 700]), ([70, 33], [70, 500]), ([24, 1, 0, 33], [4000, 10, 70, 1500])])
def test_results_may_replace_the_queries(news, lens):
    b = Batch(news, lens, 10, 2, 128, BF16, 16, seed=73).fill()
    keep, q = b.attend(0.088), b.q.cuda()
    assert b.attend(0.088, q=q, out=q) is q and torch.equal(q, keep)


def test_prompt_results_may_replace_the_queries():
    from paper_2609_37988_gb300.serving import prompt_attention
    q, k, v = (randn(gen(74), (700, h, 128), BF16) for h in (10, 2, 2))
    cu = offsets([300, 1, 33, 366])
    keep = prompt_attention(q, k, v, cu, 0.088)
    assert prompt_attention(q, k, v, cu, 0.088, out=q) is q and torch.equal(q, keep)


@pytest.mark.parametrize("news,lens", [([1, 2, 1], [300, 1, 400]), ([1, 3], [3000, 700]), ([70, 33], [70, 500]), ([24, 1, 0, 33], [4000, 10, 70, 1500])])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_queries_that_are_not_finite_reach_only_their_own_rows(news, lens, bad):
    b = Batch(news, lens, 10, 2, 128, BF16, 16, seed=79).fill()
    keep = b.attend(0.088)
    hit = [(0, 3), (sum(news) - 1, 0), (sum(news) // 2, 9)]
    for token, head in hit:
        b.q[token, head, 17] = bad
    got = b.attend(0.088)
    for token, head in hit:
        assert torch.isnan(got[token, head]).all()
        keep[token, head] = got[token, head] = 0
    assert torch.equal(got, keep)


@pytest.mark.parametrize("news,lens", [([1, 2], [300, 77]), ([40, 70], [200, 300])])
def test_limits_past_32_bits_are_no_limits(news, lens):
    from paper_2609_37988_gb300.serving import KVKError, prompt_attention
    b = Batch(news, lens, 8, 2, 64, BF16, 16, seed=80).fill()
    keep = b.attend(0.125)
    for far in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 2 ** 63 - 1):
        assert torch.equal(keep, b.attend(0.125, window=far))
        assert torch.equal(b.attend(0.125, max_new=b.n), b.attend(0.125, max_new=far))
    q, k, v = (randn(gen(81), (90, h, 64), BF16) for h in (8, 2, 2))
    own = prompt_attention(q, k, v, offsets([90]), 0.125)
    assert torch.equal(own, prompt_attention(q, k, v, offsets([90]), 0.125, window=2 ** 32 + 5))
    assert b.cache.device_error() == 0
    for back in (-1, -2 ** 32):
        with pytest.raises(KVKError):
            b.attend(0.125, window=back)
        with pytest.raises(KVKError):
            prompt_attention(q, k, v, offsets([90]), 0.125, window=back)
    for layer in (1, 2 ** 32):
        with pytest.raises(KVKError):
            b.cache.attend(layer, b.q.cuda(), b.cu, b.lengths, b.table_d, 0.125)
        with pytest.raises(KVKError):
            b.cache.append(layer, *(torch.zeros((b.n, 2, 64), dtype=BF16, device="cuda") for _ in range(2)), b.cu, b.lengths, b.table_d)


def test_attention_before_the_workspace_is_cleared_is_refused():
    """Through the C ABI, whose caller owns the workspace and orders its clearing."""
    import ctypes
    from paper_2609_37988_gb300 import _lib
    b = Batch([1, 2], [700, 300], 8, 2, 64, BF16, 16, seed=82).fill()
    so, c = _lib.load(), b.cache
    ws = torch.full_like(c.workspace, 0)  # as clear as a reset leaves it: the refusal is the host's
    h, ptr = ctypes.c_void_p(), lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    pools = [(ctypes.c_void_p * 1)(t.data_ptr()) for t in (c.k_pages[0], c.v_pages[0])]
    assert so.kvk_paged_create(ctypes.byref(c.desc), *pools, ptr(ws), ws.numel(), ctypes.byref(h)) == 0
    q, out = b.q.cuda(), torch.zeros((3, 8, 64), dtype=BF16, device="cuda")
    batch = _lib.PagedBatch(b.cu.data_ptr(), b.lengths.data_ptr(), b.table_d.data_ptr(), 2, b.table_d.shape[1], 3)
    rows = _lib.Rows(q.data_ptr(), 8 * 64, 64)
    call = lambda: so.kvk_paged_attention(h, 0, ctypes.byref(batch), ctypes.byref(rows), 0.125, 2, 0, ptr(out), None)  # noqa: E731
    torch.cuda.synchronize()
    assert call() == 1 and b"reset" in so.kvk_last_error()
    assert so.kvk_paged_reset(h, None) == 0 and call() == 0
    torch.cuda.synchronize()
    assert torch.equal(out, b.attend(0.125))
    assert so.kvk_paged_destroy(h) == 0
