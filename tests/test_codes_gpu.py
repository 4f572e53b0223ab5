"""The paged cache in 8 bits on the GPU against the float64 oracle: what an append
leaves in the pages is compared to the bit, attention within
oracle.serving.attend_bound of attention over the numbers that the pages hold (the
weights enter in f16, half a step of 2^-11, and 2^-33 of a row's largest one)."""
import math

import numpy as np
import pytest
import torch

from oracle import paged
from oracle import serving as osv
from test_serving_gpu import BF16, F16, U, close, f64, gen, ints, offsets, randn

pytestmark = pytest.mark.gpu

KIND = {BF16: "bf16", F16: "f16"}
SMALL = 2.0 ** -33


class Codes:
    """A batch over pages in 8 bits, and the same pages on the host: pools full of
    any bytes, sequences' pages in random order, the table's unused entries far
    outside the pool."""

    def __init__(self, news, lens, hq, hkv, d, dtype, page, seed=0, spare=3, slack=1, rows_behind=0, mul=1.0):
        from paper_2609_37988_gb300.serving import PagedCache
        g = gen(seed)
        self.news, self.lens, self.page, self.dtype = news, lens, page, dtype
        self.hq, self.hkv, self.d = hq, hkv, d
        per = [(max(l, 0) + page - 1) // page for l in lens]
        n_pages = sum(per) + spare
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table = np.full((len(lens), max(per + [0]) + slack), 2 ** 30, np.int64)
        for b, m in enumerate(per):
            self.table[b, :m] = [order.pop() for _ in range(m)]
        shape = (n_pages, hkv, page, d)
        self.codes = [torch.randint(0, 256, shape, generator=g, dtype=torch.int32).to(torch.uint8) for _ in range(2)]
        self.exps = [torch.randint(-128, 128, shape[:2], generator=g, dtype=torch.int32).to(torch.int8) for _ in range(2)]
        pools = [x.cuda().view(torch.float8_e4m3fn) for x in self.codes]
        exps = [x.cuda() for x in self.exps]
        self.codes, self.exps = [x.numpy() for x in self.codes], [x.numpy() for x in self.exps]
        self.cache = PagedCache(n_q_heads=hq, k_pages=pools[:1], v_pages=pools[1:], k_exps=exps[:1], v_exps=exps[1:], dtype=dtype)
        self.cu, self.lengths, self.table_d = offsets(news), ints(lens), ints(self.table.tolist())
        self.k = [(torch.randn((max(l, 0), hkv, d), generator=g) * mul).to(dtype) for l in lens]
        self.v = [(torch.randn((max(l, 0), hkv, d), generator=g) * mul).to(dtype) for l in lens]
        self.n = sum(news) + rows_behind
        self.q = torch.randn((self.n, hq, d), generator=g).to(dtype)

    def append(self, upto=None, since=None, **kw):
        """Positions since[b] .. upto[b] - 1 of every sequence, on both sides."""
        upto = [max(l, 0) for l in self.lens] if upto is None else upto
        since = [0] * len(upto) if since is None else since
        news = [u - s for u, s in zip(upto, since)]
        if sum(news):
            k, v = (torch.cat([x[s:u] for x, s, u in zip(t, since, upto)]).cuda() for t in (self.k, self.v))
            self.cache.append(0, k, v, offsets(news), ints(upto), self.table_d, **kw)
        lo, hi = paged.RANGE[KIND[self.dtype]]
        for i, x in enumerate((self.k, self.v)):
            for b, (s, u) in enumerate(zip(since, upto)):
                paged.append(self.codes[i], self.exps[i], f64(x[b][s:u]), s, self.table[b], self.page, lo, hi)
        return self

    def same(self):
        """The pools hold what the oracle's do, to the bit."""
        for pool, exps, codes, e in ((self.cache.k_pages, self.cache.k_exps, self.codes[0], self.exps[0]),
                                     (self.cache.v_pages, self.cache.v_exps, self.codes[1], self.exps[1])):
            np.testing.assert_array_equal(exps[0].cpu().numpy(), e)
            np.testing.assert_array_equal(pool[0].view(torch.uint8).cpu().numpy(), codes)
        assert self.cache.device_error() == 0
        return self

    def held(self, i, b):
        l = max(self.lens[b], 0)
        lo, hi = paged.RANGE[KIND[self.dtype]]
        return osv.from_pages(paged.values(self.codes[i], np.clip(self.exps[i], lo, hi)), self.table[b], l, self.page)

    def expected(self, scale, window):
        out, tol, at = [], [], 0
        for b, (n, l) in enumerate(zip(self.news, self.lens)):
            r = osv.attend(f64(self.q[at:at + n]), self.held(0, b), self.held(1, b), scale, window)
            if l < 0:
                r = tuple(np.zeros_like(x) for x in r)
            out.append(r[0])
            tol.append(osv.attend_bound(*r, self.d, max(l, 1), U[self.dtype], SMALL))
            if l > 0:
                # chunks: a value is code * 2^(e - E + 6) in f16, E the largest of the powers e of
                # the sequence's pages; below 2^-14 that is rounded to a multiple of 2^-24, by at most
                # 2^-25, and the weights, which sum to 1, make it at most 2^(E - 31) of the result
                pages = self.table[b, :(l + self.page - 1) // self.page]
                top = np.ldexp(1.0, self.exps[1][pages].astype(int).max(0) - 31)
                tol[-1] += np.repeat(top, self.hq // self.hkv)[:, None]
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


# -- append ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,page,hkv,d", [(BF16, 16, 2, 128), (F16, 64, 2, 64), (BF16, 128, 3, 64), (F16, 32, 4, 128), (F16, 128, 9, 128),
                                              (BF16, 16, 1, 64)])
def test_append_to_the_bit(dtype, page, hkv, d):
    b = Codes([0] * 6, [1, 5, 129, 200, 16, 0], hkv, hkv, d, dtype, page, seed=1)
    b.append().same()


@pytest.mark.parametrize("dtype,page,hkv,d", [(BF16, 16, 2, 128), (F16, 64, 2, 64), (BF16, 128, 1, 128), (F16, 32, 3, 64)])
def test_append_token_by_token_with_rising_magnitudes(dtype, page, hkv, d):
    """Codes that are there are rounded again each time a page's power rises."""
    lens = [37, 150, 3]
    b = Codes([0] * 3, lens, hkv, hkv, d, dtype, page, seed=2)
    g = gen(3)
    for x in b.k + b.v:
        x *= torch.exp2(torch.randint(-7, 5, (x.shape[0], hkv, 1), generator=g).float()).to(dtype)
    at = [0, 0, 0]
    step = 0
    while at != lens:
        step += 1
        to = [min(l, a + s) for l, a, s in zip(lens, at, ((1, 7, 0), (2, 1, 1), (1, 30, 1))[step % 3])]
        b.append(to, at)
        at = to
        if step % 5 == 0:
            b.same()
    b.same()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_append_numbers_of_every_size(dtype):
    """Zeros, the smallest and the largest numbers, numbers just at and above what a
    power holds, and what is not finite."""
    b = Codes([0] * 2, [64, 64], 2, 2, 64, dtype, 16, seed=4)
    big = torch.finfo(dtype).max
    tiny = torch.finfo(dtype).smallest_normal
    b.k[0][:16] = 0
    b.k[0][16:32, 0] = big
    b.k[0][16:32, 1] *= tiny
    b.k[0][32:48] = 448.0
    b.k[0][32, 1, 5] = 450.0 if dtype == BF16 else 448.5
    b.v[0][3, 0, 7] = float("nan")
    b.v[0][20, 1, :] = float("inf")
    b.v[0][32:48, 0] = -float("inf")
    b.v[0][50, 0, 0] = -big
    b.v[1] *= 0.0
    b.v[1][17, 1, 1] = tiny / 8
    b.append().same()
    b.append([64, 64], [63, 62]).same()


def test_append_leaves_tokens_of_no_sequence_and_the_rest_of_the_pages():
    b = Codes([0] * 2, [40, 20], 2, 2, 128, BF16, 16, seed=5)
    b.append([30, 9]).same()
    k = torch.cat([b.k[0][30:32], b.k[1][9:12], randn(gen(6), (4, 2, 128), BF16).cpu()]).cuda()
    v = torch.cat([b.v[0][30:32], b.v[1][9:12], k[5:].cpu()]).cuda()
    b.cache.append(0, k, v, ints([0, 2, 5]), ints([32, 12]), b.table_d)
    for i, x in enumerate((b.k, b.v)):
        paged.append(b.codes[i], b.exps[i], f64(x[0][30:32]), 30, b.table[0], 16, -110, 119)
        paged.append(b.codes[i], b.exps[i], f64(x[1][9:12]), 9, b.table[1], 16, -110, 119)
    b.same()
    # tokens before position 0 are not stored
    b.cache.append(0, k[:5], v[:5], ints([0, 5, 5]), ints([2, 12]), b.table_d)
    for i, x in enumerate((k, v)):
        paged.append(b.codes[i], b.exps[i], f64(x[3:5]), 0, b.table[0], 16, -110, 119)
    b.same()


@pytest.mark.parametrize("dtype,page,hq,hkv,d", [(BF16, 16, 10, 2, 128), (F16, 64, 8, 2, 64), (F16, 128, 4, 4, 128)])
@pytest.mark.parametrize("mode", ["half", "adjacent", "part", "odd strides", "own positions"])
def test_append_turns_keys_as_the_rotary_does(dtype, page, hq, hkv, d, mode):
    """To the bit: as if keys rotated by Rotary.apply had been appended."""
    from paper_2609_37988_gb300.serving import Rotary
    news, lens = [3, 0, 1, 140, 6], [3, 5, 129, 200, 4]
    g = gen(7)
    n = sum(news) + 2
    rot = Rotary(head_dim=d, rotary_dim=d // 2 + 2 if mode == "part" else d, base=1e6, adjacent=mode == "adjacent",
                 sections=None if mode == "own positions" else (d // 8, d // 8, (d // 2 + 2) // 2 - d // 4 if mode == "part" else d // 4))
    if mode == "odd strides":
        flat = randn(g, (n * (hq + 2 * hkv) * (d + 1) + 1,), dtype)[1:]
        qkv = flat.view(n, hq + 2 * hkv, d + 1)[..., :d]
    else:
        qkv = randn(g, (n, hq + 2 * hkv, d), dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    own = torch.cat([torch.arange(l - m, l) for m, l in zip(news, lens)] + [torch.zeros(2)]).to(torch.int32).cuda()
    pos = own if mode == "own positions" else torch.randint(0, 50000, (3, n), generator=g, dtype=torch.int32).cuda()
    one, two = (Codes(news, lens, hq, hkv, d, dtype, page, seed=8) for _ in range(2))
    q_out = torch.full((n, hq, d), 7.0, dtype=dtype, device="cuda")
    got = one.cache.append(0, k, v, one.cu, one.lengths, one.table_d, rotary=rot,
                           positions=None if mode == "own positions" else pos, q=q, q_out=q_out)
    q2, k2 = rot.apply(q, k, pos)
    two.cache.append(0, k2, v, two.cu, two.lengths, two.table_d)
    m = sum(news)
    assert torch.equal(got[:m], q2[:m]) and (got[m:] == 7.0).all()
    for x, y in ((one.cache.k_pages, two.cache.k_pages), (one.cache.v_pages, two.cache.v_pages)):
        assert torch.equal(x[0].view(torch.uint8), y[0].view(torch.uint8))
    assert torch.equal(one.cache.k_exps[0], two.cache.k_exps[0]) and torch.equal(one.cache.v_exps[0], two.cache.v_exps[0])
    assert one.cache.device_error() == 0


@pytest.mark.parametrize("page", [64, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_append_of_one_long_sequence_among_single_tokens(page, d):
    """Groups for few tokens go over a page's rows more than once; numbers that are not
    finite in one turn of several."""
    from paper_2609_37988_gb300.serving import Rotary
    lens = [1] * 40 + [300] + [5] * 20
    b = Codes([0] * len(lens), lens, 2, 2, d, BF16, page, seed=35)
    b.k[40][100, 1, 3] = float("inf")
    b.v[40][7, 0, 0] = float("nan")
    b.v[40][290] *= 100
    b.append().same()
    rot, pos = Rotary(head_dim=d), torch.cat([torch.arange(l) for l in lens]).to(torch.int32).cuda()
    one, two = (Codes([0] * len(lens), lens, 2, 2, d, BF16, page, seed=36) for _ in range(2))
    k, v = torch.cat(one.k).cuda(), torch.cat(one.v).cuda()
    one.cache.append(0, k, v, offsets(lens), ints(lens), one.table_d, rotary=rot)
    two.cache.append(0, rot.apply(None, k, pos)[1], v, offsets(lens), ints(lens), two.table_d)
    assert torch.equal(one.cache.k_pages[0].view(torch.uint8), two.cache.k_pages[0].view(torch.uint8))
    assert torch.equal(one.cache.k_exps[0], two.cache.k_exps[0])


@pytest.mark.parametrize("count", [33, 200])
def test_append_of_many_sequences(count):
    rng = np.random.default_rng(9)
    lens = [int(x) for x in rng.integers(0, 40, count)]
    b = Codes([0] * count, lens, 2, 2, 64, BF16, 16, seed=10)
    half = [l // 2 for l in lens]
    b.append(half).append(lens, half).same()


# -- attention ---------------------------------------------------------------------------
HEADS = [(40, 8, 128), (28, 4, 128), (8, 2, 64), (4, 4, 64), (16, 1, 128), (6, 2, 128), (48, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype,page", [(BF16, 16), (F16, 32), (BF16, 64), (F16, 128)])
def test_single_tokens(hq, hkv, d, dtype, page):
    b = Codes([1] * 7, [1, 2, 63, 64, 65, 300, 17], hq, hkv, d, dtype, page).append()
    for window in (0, 1, 50):
        b.check(window)


@pytest.mark.parametrize("news,lens", [([5, 1, 3, 0, 2], [5, 1, 130, 77, 66]), ([9, 4], [700, 4]), ([1], [2100]), ([3, 1], [1, 0]),
                                       ([2, 0, 0, 6], [513, 0, 9, 64]), ([2, 1], [1500, 1100])])
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(40, 8, 128, BF16, 16), (28, 4, 128, F16, 64), (8, 2, 64, BF16, 128), (7, 1, 128, BF16, 32)])
def test_few_tokens(news, lens, hq, hkv, d, dtype, page):
    b = Codes(news, lens, hq, hkv, d, dtype, page, seed=11).append()
    for window in (0, 1, 7, 100):
        b.check(window)
    b.check(0, max_new=sum(news))


CHUNKS = [([70, 33], [70, 500]), ([129, 1, 64, 0, 127], [129, 1, 200, 5, 383]), ([260], [260]), ([31, 300], [1000, 301]),
          ([50, 50], [20, 50]), ([9], [3000]), ([300, 7], [2500, 2100])]


@pytest.mark.parametrize("news,lens", CHUNKS)
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(10, 2, 128, BF16, 16), (7, 1, 128, F16, 32), (8, 2, 64, BF16, 64), (3, 3, 64, F16, 16),
                                                 (8, 1, 128, BF16, 128)])
def test_chunks(news, lens, hq, hkv, d, dtype, page):
    b = Codes(news, lens, hq, hkv, d, dtype, page, seed=12).append()
    for window in (0, 40, 129):
        b.check(window)


@pytest.mark.parametrize("hq,hkv,d", [(64, 1, 128), (128, 2, 64), (33, 1, 128), (51, 3, 64), (65, 65, 64)])
def test_head_groups_of_every_width(hq, hkv, d):
    b = Codes([1, 1, 1], [70, 1, 300], hq, hkv, d, BF16, 16, seed=13).append()
    b.check()
    b = Codes([9, 0, 66], [9, 5, 200], hq, hkv, d, F16, 32, seed=14).append()
    for window in (0, 50):
        b.check(window)


@pytest.mark.parametrize("news,lens", [([1, 1], [3000, 77]), ([4, 2], [1000, 130]), ([40, 130], [1000, 700]), ([700], [1500])])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_pages_that_the_window_has_left_need_no_entry(news, lens, page):
    b = Codes(news, lens, 8, 2, 128, BF16, page, seed=15).append()
    for window in (1, 33, 100, 300):
        stale = b.table.copy()
        for s, (n, m) in enumerate(zip(news, lens)):
            stale[s, :max(0, m - n - window + 1) // page] = -1 if s else 2 ** 30
        b.table_d = ints(stale.tolist())
        b.check(window)


@pytest.mark.parametrize("news", [[1, 1], [3, 2], [80, 150]])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_pages_of_very_different_powers(news, dtype):
    """Numbers from page to page a factor apart, pages of zeros among them, keys and
    values independently; queries of very different rows."""
    lens = [700, 640]
    b = Codes(news, lens, 10, 2, 128, dtype, 16, seed=16)
    g = gen(17)
    span = 30 if dtype == BF16 else 5
    for s in range(2):
        for x, lim in ((b.k[s], 3), (b.v[s], span)):
            e = torch.randint(-lim, lim + 1, (len(x) // 16 + 1, 2, 1), generator=g).float()
            e[::7] = -200.0  # zeros
            x *= torch.exp2(e).repeat_interleave(16, 0)[: len(x)].to(dtype)
    b.q *= torch.exp2(torch.randint(-6, 3, (b.n, 10, 1), generator=g).float()).to(dtype)
    b.append().same()
    for window in (0, 33):
        b.check(window)


@pytest.mark.parametrize("news", [[1, 2], [70, 90]])
def test_far_powers_of_bf16(news):
    """All values of a sequence near the ends of the range, keys and queries such
    that scores are ordinary."""
    b = Codes(news, [300, 200], 8, 2, 64, BF16, 32, seed=18)
    for s, e in enumerate((100.0, -90.0)):
        b.v[s] *= 2.0 ** e
        b.k[s] *= 2.0 ** (e / 2)
        at = slice(0, news[0]) if s == 0 else slice(news[0], None)
        b.q[at] *= 2.0 ** (-e / 2)
    b.append().same()
    b.check()


@pytest.mark.parametrize("news", [[1, 1], [3, 2], [80, 150]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(news, bad):
    lens = [200, 190]
    b = Codes(news, lens, 10, 2, 128, BF16, 16, seed=19)
    for s, t, ch in [(0, lens[0] - 1, 3), (1, lens[1] - 2, 77), (1, lens[1] - news[1] // 2 - 1, 5), (0, 60, 100)]:
        b.v[s][t, 1, ch] = bad
    b.k[1][lens[1] - 1, 0, 9] = float("nan")
    b.append().same()
    for window in (0, 60):
        scale = 1.0 / math.sqrt(128)
        got = f64(b.attend(scale, window)[: sum(news)])
        ref, tol = b.expected(scale, window)
        fine = np.isfinite(ref)
        assert (np.isfinite(got) == fine).all()
        assert (np.abs(got - ref)[fine] <= tol[fine]).all()


@pytest.mark.parametrize("news", [[2], [90]])
def test_queries_that_are_not_finite_spoil_their_rows_alone(news):
    b = Codes(news, [300], 4, 2, 128, BF16, 16, seed=20).append()
    keep = f64(b.attend(0.088))
    b.q[0, 1, 5] = float("nan")
    b.q[1, 2, 0] = float("inf")
    got = f64(b.attend(0.088))
    spoilt = np.zeros(got.shape[:2], bool)
    spoilt[0, 1] = spoilt[1, 2] = True
    assert not np.isfinite(got[spoilt]).any()
    np.testing.assert_array_equal(got[~spoilt], keep[~spoilt])


@pytest.mark.parametrize("news,lens", [([4, 1, 1], [3000, 1000, 700]), ([40, 1, 100], [3000, 1000, 700])])
def test_strided_queries_and_repeated_calls_agree_to_the_bit(news, lens):
    b = Codes(news, lens, 28, 4, 128, BF16, 32, seed=21).append()
    wide = torch.zeros((b.n, 40, 128), dtype=BF16, device="cuda")
    wide[:, 5:33] = b.q.cuda()
    for max_new in (None, b.n):
        first = b.attend(0.088, max_new=max_new)
        assert torch.equal(first, b.attend(0.088, max_new=max_new, q=wide[:, 5:33]))
        perm = b.q.cuda().permute(1, 0, 2).contiguous().permute(1, 0, 2)  # heads outermost
        assert torch.equal(first, b.attend(0.088, max_new=max_new, q=perm))
        for _ in range(5):
            assert torch.equal(first, b.attend(0.088, max_new=max_new))
        own = b.q.cuda()
        assert b.attend(0.088, max_new=max_new, q=own, out=own) is own and torch.equal(first, own)


def test_rows_in_no_sequence_stay_and_empty_batches():
    b = Codes([3, 2], [70, 9], 8, 2, 64, BF16, 16, rows_behind=4, seed=22).append()
    for max_new in (3, b.n):
        out = torch.full((b.n, 8, 64), 7.0, dtype=BF16, device="cuda")
        b.attend(0.125, out=out, max_new=max_new)
        assert (out[5:] == 7.0).all() and not (out[:5] == 7.0).all()
    e = Codes([0, 0], [0, 40], 8, 2, 64, BF16, 16, seed=23).append()
    assert e.attend(0.125).shape == (0, 8, 64)
    q = torch.full((3, 8, 64), 5.0, dtype=BF16, device="cuda")
    assert (e.attend(0.125, q=q, out=q.clone(), max_new=3) == 5.0).all()
    assert b.cache.device_error() == e.cache.device_error() == 0


@pytest.mark.parametrize("count", [33, 130])
@pytest.mark.parametrize("most", [1, 3, 40])
def test_many_sequences(count, most):
    rng = np.random.default_rng(24)
    news = [int(x) for x in rng.integers(0, most + 1, count)]
    lens = [int(x) for x in rng.integers(0, 70, count)]
    Codes(news, lens, 10, 2, 64, BF16, 16, seed=25).append().check(25)


def test_device_errors_and_recovery():
    b = Codes([1, 2], [80, 90], 8, 2, 64, BF16, 16, seed=26, slack=0).append()
    keep = b.attend(0.125)
    bad = b.table_d.clone()
    for entry in (10 ** 6, -5):
        bad[0, 2] = entry
        for max_new in (2, 30):
            b.cache.attend(0, b.q.cuda(), b.cu, b.lengths, bad, 0.125, max_new=max_new)
            assert b.cache.device_error() == 32
    b.attend(0.125, max_new=1)
    assert b.cache.device_error() == 4
    b.cache.attend(0, b.q.cuda(), b.cu, ints([80, 10 ** 6]), b.table_d, 0.125, max_new=2)
    assert b.cache.device_error() == 4
    k = torch.zeros((3, 2, 64), dtype=BF16, device="cuda")
    b.cache.append(0, k, k, b.cu, ints([80, 10 ** 6]), b.table_d)
    assert b.cache.device_error() == 2
    b.cache.append(0, k, k, b.cu, ints([49, 90]), torch.full_like(b.table_d, 10 ** 6))
    assert b.cache.device_error() == 32
    b.append()
    assert torch.equal(keep, b.attend(0.125)) and b.cache.device_error() == 0


@pytest.mark.parametrize("news,lens", [([1, 1, 1], [500, 2, 77]), ([64, 200], [64, 900]), ([40, 20], [3000, 2200])])
def test_captured_and_replayed_as_lengths_grow(news, lens):
    """An append and an attention in one graph; the lengths are read when it runs."""
    b = Codes(news, lens, 10, 2, 128, BF16, 16, seed=27)
    scale = 1.0 / math.sqrt(128)
    start = [l - n - 2 * n if l > 3 * n else 0 for n, l in zip(news, lens)]
    b.append(start)
    side = torch.cuda.Stream()
    n = sum(news)
    k, v, q = (torch.zeros((n, h, 128), dtype=BF16, device="cuda") for h in (2, 2, 10))
    out = torch.empty_like(q)
    b.cache.attend(0, q, b.cu, b.lengths, b.table_d, scale, max_new=max(news))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.cache.append(0, k, v, b.cu, b.lengths, b.table_d)
        b.attend(scale, q=q, out=out)
    q.copy_(b.q)
    at, full = start, lens
    for _ in range(3):
        to = [a + m for a, m in zip(at, news)]
        if any(t > l for t, l in zip(to, full)):
            break
        k.copy_(torch.cat([x[a:t] for x, a, t in zip(b.k, at, to)]))
        v.copy_(torch.cat([x[a:t] for x, a, t in zip(b.v, at, to)]))
        b.lengths.copy_(ints(to))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        lo, hi = paged.RANGE["bf16"]
        for i, x in enumerate((b.k, b.v)):
            for s, (a, t) in enumerate(zip(at, to)):
                paged.append(b.codes[i], b.exps[i], f64(x[s][a:t]), a, b.table[s], 16, lo, hi)
        b.lens = to
        ref, tol = b.expected(scale, 0)
        close(out, ref, tol, f"lengths {to}")
        b.same()
        at = to
    assert at != start


@pytest.mark.parametrize("news", [[1, 2], [40, 70]])
def test_pools_past_two_to_the_31_elements(news):
    from paper_2609_37988_gb300.serving import PagedCache
    hq, hkv, d, page = 8, 8, 128, 128
    n_pages = 2 ** 31 // (hkv * page * d) + 4
    cache = PagedCache(n_q_heads=hq, n_kv_heads=hkv, n_layers=1, head_dim=d, n_pages=n_pages, page_size=page, dtype=BF16, bits=8)
    lens = [300, 200]
    table = np.array([[n_pages - 1, 0, n_pages - 3], [n_pages - 2, 1, 0]])
    small = np.array([[5, 0, 3], [4, 1, 0]])  # the same pages, counted from one less
    g = gen(28)
    k, v = ([torch.randn((l, hkv, d), generator=g).to(BF16) for l in lens] for _ in range(2))
    q = torch.randn((sum(news), hq, d), generator=g).to(BF16)
    cache.append(0, torch.cat(k).cuda(), torch.cat(v).cuda(), offsets(lens), ints(lens), ints(table.tolist()))
    got = cache.attend(0, q.cuda(), offsets(news), ints(lens), ints(table.tolist()), 0.088, max_new=max(news))
    pools = []
    for x in (k, v):
        codes, exps = np.zeros((6, hkv, page, d), np.uint8), np.zeros((6, hkv), np.int8)
        for s in range(2):
            paged.append(codes, exps, f64(x[s]), 0, small[s], page, -110, 119)
        pools.append(paged.values(codes, exps))
    at = 0
    for b, n in enumerate(news):
        r = osv.attend(f64(q[at:at + n]), *(osv.from_pages(x, small[b], lens[b], page) for x in pools), 0.088)
        close(got[at:at + n], r[0], osv.attend_bound(*r, d, lens[b], U[BF16], SMALL))
        at += n
    assert cache.device_error() == 0


def test_two_caches_at_once():
    a = Codes([1, 2, 1], [900, 300, 5], 10, 2, 128, BF16, 16, seed=29).append()
    b = Codes([30, 80], [700, 900], 10, 2, 128, BF16, 16, seed=30).append()
    keep_a, keep_b = a.attend(0.088), b.attend(0.088)
    qa, qb = a.q.cuda(), b.q.cuda()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(10):
        outs.append((keep_a, a.attend(0.088, q=qa, stream=streams[0])))
        outs.append((keep_b, b.attend(0.088, q=qb, stream=streams[1])))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in outs)


@pytest.mark.parametrize("gap", [12.0, 17.5, 20.0])
@pytest.mark.parametrize("dtype,d,page,positions", [(F16, 128, 16, 4096), (BF16, 64, 128, 4096), (BF16, 128, 32, 400)])
def test_weights_far_below_the_largest(gap, dtype, d, page, positions):
    """One key `gap` above all the others, its value zero: the result is what the
    others' small weights bring."""
    b = Codes([1], [positions], 2, 1, d, dtype, page, seed=31, rows_behind=20)
    b.q.zero_()
    b.q[..., 0] = 1.0
    b.k[0].zero_()
    b.k[0][positions // 3, 0, 0] = gap
    b.v[0][:] = 1024.0 + 4 * torch.arange(d)
    b.v[0][positions // 3] = 0.0
    b.append()
    r = osv.attend(f64(b.q[:1]), b.held(0, 0), b.held(1, 0), 1.0)
    for max_new in (1, b.n):
        got = b.attend(1.0, max_new=max_new)[:1]
        close(got, r[0], osv.attend_bound(*r, d, positions, U[dtype], SMALL), f"max_new {max_new}")


@pytest.mark.parametrize("news", [[2, 1], [80, 150]])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_keys_of_zeros_and_small_queries(news, dtype):
    """Pages of zero keys have the least power; scores of 0 and masked ones beside each other."""
    b = Codes(news, [200, 190], 10, 2, 128, dtype, 16, seed=32)
    for s in range(2):
        b.k[s][: 160 + 20 * s] = 0.0
    b.q *= 2.0 ** (-60 if dtype == BF16 else -12)
    b.append().same()
    for window in (0, 33):
        b.check(window)


@pytest.mark.parametrize("news", [[1, 1], [70, 130]])
def test_an_attention_that_gives_up_says_so(news):
    b = Codes(news, [200, 190], 10, 2, 128, BF16, 16, seed=33).append()
    keep = b.attend(0.088)
    b.cache.set_give_up(True)
    b.attend(0.088)
    assert b.cache.device_error() == 8
    b.cache.set_give_up(False)
    assert torch.equal(b.attend(0.088), keep) and b.cache.device_error() == 0


@pytest.mark.parametrize("new", [1, 3, 20])
def test_contexts_of_seventy_thousand_positions(new):
    """A table wider than 65536 positions, pieces in every CTA; a window at its end."""
    b = Codes([new], [70001], 4, 1, 64, F16, 16, seed=34).append()
    for window in (0, 66000):
        b.check(window)


# -- chunks of one query tile: the two softmax groups share its tiles of positions ------
ONE_TILE = [([17, 18, 5], [17, 1290, 128]), ([18], [2049]), ([4, 9, 18], [256, 384, 129]), ([18, 0, 12], [9, 0, 1500]), ([6] * 9, [640] * 9)]


@pytest.mark.parametrize("news,lens", ONE_TILE)
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(40, 8, 128, BF16, 16), (28, 4, 128, F16, 64), (8, 2, 64, BF16, 128), (1, 1, 64, F16, 16)])
def test_chunks_of_one_query_tile(news, lens, hq, hkv, d, dtype, page):
    b = Codes(news, lens, hq, hkv, d, dtype, page, seed=35).append()
    for window in (0, 1, 40, 129, 300):
        b.check(window)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_one_query_tile_over_pages_of_very_different_powers(dtype):
    test_pages_of_very_different_powers([9, 14], dtype)
    test_keys_of_zeros_and_small_queries([9, 14], dtype)


def test_one_query_tile_over_far_powers():
    test_far_powers_of_bf16([20, 30])


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("rising", [True, False])
def test_one_query_tile_with_weights_and_values_in_every_other_tile(page, rising):
    """Scores and values of the even tiles of positions far from those of the odd ones."""
    b = Codes([20], [700], 4, 1, 128, BF16, page, seed=36)
    tile = torch.arange(700) // 128
    b.k[0] *= torch.exp2(((tile % 2 == 0) == rising).float() * 3)[:, None, None].to(BF16)
    b.v[0] *= torch.exp2((tile % 2 == (1 if rising else 0)).float() * 40)[:, None, None].to(BF16)
    b.append().same()
    for window in (0, 128, 300):
        b.check(window)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_one_query_tile_with_values_that_are_not_finite(bad):
    test_values_that_are_not_finite_reach_only_rows_that_see_them([20, 12], bad)
    test_queries_that_are_not_finite_spoil_their_rows_alone([40])


@pytest.mark.parametrize("news,lens", [([18, 1, 7], [3000, 1000, 700]), ([7] * 20, [500] * 20)])
def test_one_query_tile_repeated_strided_and_captured(news, lens):
    test_strided_queries_and_repeated_calls_agree_to_the_bit(news, lens)
    test_captured_and_replayed_as_lengths_grow(news, lens)


def test_more_tokens_than_said_of_one_query_tile():
    """Refused by the device's own check; what is read and written stays in bounds and
    later calls are as before."""
    b = Codes([60, 9], [300, 90], 10, 2, 128, BF16, 16, seed=37).append()
    keep = b.attend(0.088)
    b.attend(0.088, max_new=9)
    assert b.cache.device_error() == 4
    assert torch.equal(b.attend(0.088), keep) and b.cache.device_error() == 0


def test_one_query_tile_that_gives_up_says_so():
    test_an_attention_that_gives_up_says_so([20, 7])


# -- few tokens: what enters the weights ---------------------------------------------------
def few_bound(b, r, s):
    """oracle.serving.attend_bound for up to 16 rows of a KV head: weights are rounded to f16
    (half a step of 2^-11), kept 2^14 times as large as a row's largest and times 2^(e - E) of
    their page's power against the largest of the pages that are seen; what f16 cuts off, half
    of 2^-24, is 2^-39 * 2^(E - e) of the row's largest.  No term of f16 tiles of values."""
    l = max(b.lens[s], 1)
    pages = b.table[s, :(l + b.page - 1) // b.page]
    e = b.exps[1][pages].astype(int)
    smallest = 2.0 ** (e.max() - e.min() - 39)
    return osv.attend_bound(*r, b.d, l, 2.0 ** -11, smallest) + U[b.dtype] * np.abs(r[0]) * (1 + U[b.dtype])


# odd and even numbers of pages, ends in either half of a warp's 32 positions
SHORT = [1, 16, 17, 33, 48, 80, 100, 144, 300, 305, 400]
LONG = [529, 545, 1100, 1300, 2060]


@pytest.mark.parametrize("lens", [SHORT, LONG])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hq,hkv,d,new,dtype", [(8, 2, 64, 1, BF16), (8, 2, 64, 4, BF16), (40, 8, 128, 1, BF16), (40, 8, 128, 3, BF16),
                                                (7, 1, 128, 2, BF16), (28, 4, 128, 1, F16)])
def test_few_tokens_over_small_values(lens, page, hq, hkv, d, new, dtype):
    """Positions that no row sees, behind a context or before its window, bring no power
    into the weights of those that are seen, however small their values are."""
    b = Codes([min(new, l) for l in lens], lens, hq, hkv, d, dtype, page, seed=38)
    for s, x in enumerate(b.v):
        x *= 2.0 ** ((-90, -30, -60, -20) if dtype == BF16 else (-8, -4, -6, -2))[s % 4]
    b.append().same()
    scale = 1.0 / math.sqrt(d)
    for window in (0, 5, 33, 200):
        got, at = f64(b.attend(scale, window)), 0
        for s, n in enumerate(b.news):
            r = osv.attend(f64(b.q[at:at + n]), b.held(0, s), b.held(1, s), scale, window)
            close(got[at:at + n], r[0], few_bound(b, r, s), f"window {window}, {b.lens[s]} positions")
            at += n
    assert b.cache.device_error() == 0


@pytest.mark.parametrize("new", [1, 3, 20, 60])
@pytest.mark.parametrize("qe,ke", [(100, 100), (120, 60), (60, 120), (126, 126), (-120, 118)])
def test_scores_of_zero_between_numbers_at_the_ends_of_bf16(new, qe, ke):
    """Queries and keys whose powers multiply past binary32, in different channels: all
    scores are 0, and every position that is seen has the same weight."""
    b = Codes([new, 1], [100, 77], 8, 2, 64, BF16, 16, seed=39)
    b.q.zero_()
    b.q[..., 0] = 2.0 ** qe
    for x in b.k:
        x.zero_()
        x[..., 1] = 2.0 ** ke
    b.append().same()
    for window in (0, 33):
        b.check(window)
