"""Copying, forking and compacting pages on the GPU against oracle.paged, to the bit,
and a run of the operators together."""
import math

import numpy as np
import pytest
import torch

from oracle import paged
from oracle import serving as osv
from test_serving_gpu import BF16, F16, U, close, f64, gen, ints, offsets, randn

pytestmark = pytest.mark.gpu


class Pool:
    """Pools of random content, in 8 or 16 bits, and what they are expected to hold."""

    def __init__(self, n_pages, page, bits, layers=2, hkv=2, d=64, seed=0):
        from paper_2609_37988_gb300.serving import PagedCache
        self.cache = PagedCache(n_q_heads=hkv, n_layers=layers, n_kv_heads=hkv, head_dim=d, n_pages=n_pages, page_size=page, bits=bits)
        self.n, self.page, self.bits = n_pages, page, bits
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in self.tensors():
            t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
        self.want = [t.clone() for t in self.tensors()]

    def tensors(self):
        c = self.cache
        return [t.view(torch.uint8).view(self.n, -1) for t in c.k_pages + c.v_pages + (c.k_exps + c.v_exps if self.bits == 8 else [])]

    def moved(self, pairs):
        """Pages copied, all read before any is written."""
        pairs = [(a, b) for a, b in pairs if b >= 0]
        if pairs:
            a, b = (torch.tensor(x, device="cuda") for x in zip(*pairs))
            for w in self.want:
                w[b] = w[a]
        for t, w in zip(self.tensors(), self.want):
            assert torch.equal(t, w)
        assert self.cache.device_error() == 0


def table_of(g, n_pages, page, lens, width, shared=0):
    """(refs, table): pages in random order; `shared` rows begin with another's."""
    order = list(g.permutation(n_pages))
    table, refs = np.full((len(lens), width), -77), np.zeros(n_pages, int)
    for b, l in enumerate(lens):
        m = (l + page - 1) // page
        for j in range(m):
            if b and b <= shared and j < (min(l, lens[b - 1]) // page):
                table[b, j] = table[b - 1, j]
            else:
                table[b, j] = order.pop()
            refs[table[b, j]] += 1
    return refs, table


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("page,layers,hkv,d", [(16, 2, 2, 64), (32, 3, 1, 128), (128, 1, 5, 128), (16, 1, 1, 64)])
def test_copy(bits, page, layers, hkv, d):
    p = Pool(23, page, bits, layers, hkv, d)
    p.cache.copy(ints([3, -1, 22, 5]), ints([7, 8, 0, -1]))
    p.moved([(3, 7), (22, 0)])
    p.cache.copy(ints([]), ints([]))
    p.cache.copy(ints([4]), ints([4]))
    p.moved([])
    for bad in (([23], [0]), ([0], [23]), ([-2], [0]), ([0], [2 ** 31 - 1])):
        p.cache.copy(ints(bad[0]), ints(bad[1]))
        assert p.cache.device_error() == 32
    p.moved([])


def test_copy_of_more_layers_than_one_launch_takes():
    p = Pool(9, 16, 8, layers=200, hkv=1)
    p.cache.copy(ints([1, 2]), ints([5, 6]))
    p.moved([(1, 5), (2, 6)])


def test_copy_past_two_to_the_31_bytes():
    p = Pool(9000, 128, 16, layers=1, hkv=8, d=128)
    p.cache.copy(ints([8999, 3]), ints([0, 8998]))
    p.moved([(8999, 0), (3, 8998)])


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("seed", range(12))
def test_fork(bits, seed):
    """Rows of any parents, shorter and longer; pages that others hold too."""
    g = np.random.default_rng(seed)
    page = int(g.choice([16, 32, 64, 128]))
    B, R, width = int(g.integers(0, 9)), int(g.integers(0, 14)), 9
    lens = [int(g.integers(0, 6 * page)) for _ in range(B)]
    n_pages = 9 * (B + R) + 6 + (3000 if seed % 3 == 0 else 0)
    refs, table = table_of(g, n_pages, page, lens, width, shared=2)
    for x in g.integers(0, n_pages, 5):  # held by others
        refs[x] += 1
    parents = [int(x) for x in g.integers(-1, B, R)] if B else [-1] * R
    held = [lens[p] if p >= 0 else 0 for p in parents]
    after = [int(g.choice([h, h + 1, max(0, h - int(g.integers(0, page))), h // 2, int(g.integers(0, width * page + 1))])) for h in held]
    pool = Pool(n_pages, page, bits)
    refs2, out, copies, short = paged.fork(refs, table, lens, parents, after, width, page)
    assert short == 0
    args = ints(refs.tolist()), ints(table.tolist()).view(B, width), ints(lens)
    got_refs, got = pool.cache.fork(*args, ints(parents), ints(after))
    np.testing.assert_array_equal(got.cpu().numpy(), out)
    np.testing.assert_array_equal(got_refs.cpu().numpy(), refs2)
    pool.moved(copies)
    # lengths of the parents, a wider table, the counts in place
    refs2, out, copies, short = paged.fork(refs, table, lens, parents, None, width + 2, page)
    mine = ints(refs.tolist())
    to = torch.full((R, width + 2), 5, dtype=torch.int32, device="cuda")
    assert pool.cache.fork(mine, *args[1:], ints(parents), out=(mine, to))[0] is mine
    np.testing.assert_array_equal(to.cpu().numpy(), out)
    np.testing.assert_array_equal(mine.cpu().numpy(), refs2)
    pool.moved(copies)
    # all let go
    refs2, _, _, _ = paged.fork(refs, table, lens, [], [], 0, page)
    np.testing.assert_array_equal(pool.cache.free(*args).cpu().numpy(), refs2)
    pool.moved([])


def test_fork_of_a_large_batch():
    """Many rows, pools of many chunks, a row that takes more pages than a chunk has."""
    g = np.random.default_rng(40)
    page, B, width = 16, 300, 2100
    lens = [int(g.integers(1, 900)) for _ in range(B)]
    refs, table = table_of(g, 40000, page, lens, width)
    parents = [int(x) for x in g.integers(0, B, B)]
    parents[7] = -1
    after = [lens[p] + 1 if p >= 0 else 32000 for p in parents]
    pool = Pool(40000, page, 8, layers=1, hkv=1)
    refs2, out, copies, short = paged.fork(refs, table, lens, parents, after, width, page)
    args = ints(refs.tolist()), ints(table.tolist()), ints(lens), ints(parents), ints(after)
    got_refs, got = pool.cache.fork(*args)
    np.testing.assert_array_equal(got.cpu().numpy(), out)
    np.testing.assert_array_equal(got_refs.cpu().numpy(), refs2)
    assert short == 0 and len(copies) > 50
    pool.moved(copies)
    for _ in range(3):
        again = pool.cache.fork(*args)
        assert torch.equal(again[0], got_refs) and torch.equal(again[1], got)


def test_fork_without_pages_left_and_of_what_is_no_row():
    page = 16
    pool = Pool(4, page, 16)
    refs, table = ints([1, 1, 0, 1]), ints([[0, 1, 7], [3, -5, -5]])
    r, t = pool.cache.fork(refs, table, ints([20, 5]), ints([0, 0, 1]), ints([33, 40, 5]))
    assert pool.cache.device_error() == 2
    # row 0 keeps page 1 and gets page 2; row 1 gets neither its copy nor another
    assert t.tolist() == [[0, 1, 2], [0, -1, -1], [3, -1, -1]] and r.tolist() == [2, 1, 1, 1]
    pool.moved([])
    r, t = pool.cache.fork(refs, table, ints([20, 5]), ints([5, -3, 1]), ints([0, 4, 5]))
    assert pool.cache.device_error() == 4 and t.tolist() == [[-1] * 3, [2, -1, -1], [3, -1, -1]] and r.tolist() == [0, 0, 1, 1]
    for lens, after, code in (([20, 500], [5], 4), ([20, 5], [-1], 4), ([20, 5], [500], 6), ([48, 5], [48], 32)):
        pool.cache.fork(refs, table, ints(lens), ints([0]), ints(after))
        assert pool.cache.device_error() & code, (lens, after)
    # a row's page that nobody is counted for
    pool.cache.fork(ints([0, 1, 0, 1]), table, ints([20, 5]), ints([0, 1]))
    assert pool.cache.device_error() == 4


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("seed", range(10))
def test_compact(bits, seed):
    g = np.random.default_rng(seed + 100)
    page = int(g.choice([16, 32, 64, 128]))
    B, width = int(g.integers(0, 9)), 9
    lens = [int(g.integers(0, 9 * page + 1)) for _ in range(B)]
    n_pages = [1, 9 * B + 7, 2500, 1024, 90][seed % 5] + (9 * B if seed % 5 in (0, 4) else 0)
    refs, table = table_of(g, n_pages, page, lens, width, shared=2)
    for x in g.integers(0, n_pages, [0, 3, 900, n_pages, 0][seed % 5]):
        refs[x] += 1
    pool = Pool(n_pages, page, bits)
    refs2, out, where, moves = paged.compact(refs, table, lens, page)
    used = ints([-1])
    args = ints(refs.tolist()), ints(table.tolist()).view(B, width), ints(lens)
    got_refs, got, got_where = pool.cache.compact(*args, used=used)
    np.testing.assert_array_equal(got.cpu().numpy(), out)
    np.testing.assert_array_equal(got_refs.cpu().numpy(), refs2)
    np.testing.assert_array_equal(got_where.cpu().numpy(), where)
    assert int(used) == (refs > 0).sum()
    pool.moved(moves)
    # in place; nothing is left to move
    mine, t = args[0].clone(), args[1].clone()
    pool.cache.compact(mine, t, args[2], out=(mine, t, got_where))
    assert torch.equal(mine, got_refs) and torch.equal(t, got)
    pool.moved(moves)
    again = pool.cache.compact(got_refs, got, args[2])
    assert torch.equal(again[0], got_refs) and torch.equal(again[1], got)
    pool.moved([])


def test_compact_of_a_large_pool_and_errors():
    g = np.random.default_rng(77)
    refs = (g.random(70001) < 0.3).astype(int) * 2
    pool = Pool(70001, 16, 8, layers=1, hkv=1)
    refs2, _, where, moves = paged.compact(refs, np.zeros((0, 3)), [], 16)
    none = torch.zeros((0, 3), dtype=torch.int32, device="cuda"), ints([])
    got_refs, _, got_where = pool.cache.compact(ints(refs.tolist()), *none)
    np.testing.assert_array_equal(got_refs.cpu().numpy(), refs2)
    np.testing.assert_array_equal(got_where.cpu().numpy(), where)
    pool.moved(moves)
    small = Pool(4, 16, 16)
    for table, lens, code in (([[9, 1]], [5], 32), ([[2, 1]], [5], 4), ([[0, 1]], [500], 4)):
        small.cache.compact(ints([1, 1, 0, 1]), ints(table), ints(lens))
        assert small.cache.device_error() == code


def test_fork_and_compact_of_more_layers_than_one_launch_takes():
    page, g = 16, np.random.default_rng(9)
    lens = [20, 40, 5]
    refs, table = table_of(g, 40, page, lens, 4)
    pool = Pool(40, page, 8, layers=130, hkv=1)
    refs2, out, copies, _ = paged.fork(refs, table, lens, [0, 0, 1], [21, 22, 41], 4, page)
    got_refs, got = pool.cache.fork(ints(refs.tolist()), ints(table.tolist()), ints(lens), ints([0, 0, 1]), ints([21, 22, 41]))
    np.testing.assert_array_equal(got.cpu().numpy(), out)
    pool.moved(copies)
    refs3, out3, where, moves = paged.compact(refs2, out, [21, 22, 41], page)
    r, t, w = pool.cache.compact(got_refs, got, ints([21, 22, 41]))
    for x, y in ((r, refs3), (t, out3), (w, where)):
        np.testing.assert_array_equal(x.cpu().numpy(), y)
    pool.moved(moves)


@pytest.mark.parametrize("call", ["fork", "compact", "copy"])
def test_on_another_stream(call):
    """Outputs and copies are there once that stream has run."""
    page, g = 16, np.random.default_rng(10)
    lens = [200, 47]
    refs, table = table_of(g, 60, page, lens, 14)
    pool = Pool(60, page, 16)
    args = ints(refs.tolist()), ints(table.tolist()), ints(lens)
    parents, src, dst = ints([1, 1, 0]), ints([3]), ints([59])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    if call == "fork":
        got = pool.cache.fork(*args, parents, stream=side)
        want = paged.fork(refs, table, lens, [1, 1, 0], None, 14, page)
    elif call == "compact":
        got = pool.cache.compact(*args, stream=side)
        want = paged.compact(refs, table, lens, page)
    else:
        pool.cache.copy(src, dst, stream=side)
        got, want = (), ([(3, 59)],)
    side.synchronize()
    for x, y in zip(got, want):
        np.testing.assert_array_equal(x.cpu().numpy(), y)
    pool.moved([m for m in want if isinstance(m, list)][0])


def test_captured_forks_follow_their_inputs():
    """Fork, compaction and copy in one graph, replayed with other tables."""
    page, width, n_pages = 16, 6, 80
    pool = Pool(n_pages, page, 8)
    refs, table = torch.zeros(n_pages, dtype=torch.int32, device="cuda"), torch.zeros((4, width), dtype=torch.int32, device="cuda")
    lens, parents, after = (torch.zeros(4, dtype=torch.int32, device="cuda") for _ in range(3))
    mid, end = (torch.zeros_like(refs), torch.zeros_like(table)), (torch.zeros_like(refs), torch.zeros_like(table), torch.zeros_like(refs))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        pool.cache.fork(refs, table, lens, parents, after, out=mid)
        pool.cache.compact(*mid, after, out=end)
    for seed in range(4):
        g = np.random.default_rng(seed + 200)
        l = [int(g.integers(0, 5 * page)) for _ in range(4)]
        r, t = table_of(g, n_pages, page, l, width)
        p = [int(x) for x in g.integers(-1, 4, 4)]
        a = [int(g.integers(0, 6 * page)) for _ in range(4)]
        for x, y in ((refs, r), (table, t), (lens, l), (parents, p), (after, a)):
            x.copy_(torch.as_tensor(np.asarray(y), dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        r2, t2, copies, _ = paged.fork(r, t, l, p, a, width, page)
        r3, t3, where, moves = paged.compact(r2, t2, a, page)
        for x, y in zip(end, (r3, t3, where)):
            np.testing.assert_array_equal(x.cpu().numpy(), y)
        pairs = [(x, y) for x, y in copies if y >= 0]
        for w in pool.want:
            for x, y in pairs:
                w[y] = w[x]
        pool.moved(moves)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(10, 2, 128, BF16, 16), (8, 2, 64, F16, 64)])
def test_prompts_then_beams_then_a_compaction(bits, hq, hkv, d, dtype, page):
    """Prompts enter pages that a fork hands out, beams go on from them token by
    token and change places, a prompt ends, the pool is compacted: every step's
    attention against the oracle's over what the sequence's own tokens were."""
    from paper_2609_37988_gb300.serving import PagedCache, Rotary
    g, rng = gen(50), np.random.default_rng(51)
    prompts, beams, n_pages, width = [45, 130], 3, 90, 14
    cache = PagedCache(n_layers=3, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, n_pages=n_pages, page_size=page, dtype=dtype, bits=bits)
    rot, scale = Rotary(head_dim=d, base=1e6), 1.0 / math.sqrt(d)
    layer, kind = 2, "bf16" if dtype == BF16 else "f16"
    lo, hi = paged.RANGE[kind]
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    none = torch.zeros((0, width), dtype=torch.int32, device="cuda"), ints([])
    held = list(prompts)
    refs, table = cache.fork(refs, *none, ints([-1, -1]), ints(held))
    # each row's history: what went into the cache, in calls
    history = [[] for _ in held]

    def held_of(calls):
        """Keys and values as the pages hold them after these calls: a page's codes
        are rounded again as its power rises."""
        out = []
        for x in (0, 1):
            whole = np.concatenate([c[x] for c in calls])
            n = len(whole)
            if bits == 16:
                out.append(np.transpose(whole, (1, 0, 2)))
                continue
            m = (n + page - 1) // page
            codes, exps, at = np.zeros((m, hkv, page, d), np.uint8), np.zeros((m, hkv), np.int8), 0
            for c in calls:
                paged.append(codes, exps, c[x], at, np.arange(m), page, lo, hi)
                at += len(c[x])
            out.append(osv.from_pages(paged.values(codes, exps), np.arange(m), n, page))
        return out

    def step(news):
        n = sum(news)
        qkv = randn(g, (n, hq + 2 * hkv, d), dtype)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        cu, lengths = offsets(news), ints(held)
        qr = cache.append(layer, k, v, cu, lengths, table, rotary=rot, q=q)
        pos = ints(np.concatenate([np.arange(h - m, h) for m, h in zip(news, held)]).tolist())
        q2, k2 = rot.apply(q, k, pos)
        assert torch.equal(qr, q2)
        out = cache.attend(layer, qr, cu, lengths, table, scale, max_new=max(news))
        at = 0
        for b, m in enumerate(news):
            rows = slice(at, at + m)
            history[b] = history[b] + [(f64(k2[rows]), f64(v[rows]))]
            r = osv.attend(f64(qr[rows]), *held_of(history[b]), scale)
            close(out[rows], r[0], osv.attend_bound(*r, d, held[b], U[dtype], 2.0 ** -33), f"row {b}")
            at += m

    step(prompts)
    parents = [0] * beams + [1] * beams
    for turn in range(7):
        after = [held[p] + 1 for p in parents]
        refs, table = cache.fork(refs, table, ints(held), ints(parents), ints(after))
        history, held = [history[p] for p in parents], after
        step([1] * len(held))
        parents = [int(x) for x in (rng.integers(0, beams, beams)).tolist() + (beams + rng.integers(0, beams, len(held) - beams)).tolist()]
        if turn == 3:  # a drafted token too many is taken back
            held = [h - 1 for h in held]
            refs, table = cache.fork(refs, table, ints([h + 1 for h in held]), ints(list(range(len(held)))), ints(held))
            history = [x[:-1] for x in history]
            if bits == 8:
                break  # a page's power may stay higher: the next steps are the other test's
        if turn == 4:
            refs, table, where = cache.compact(refs, table, ints(held))
            u = int((refs > 0).sum())
            assert bool((refs[:u] > 0).all())
    counts = torch.bincount(table[table >= 0].long(), minlength=n_pages).to(torch.int32)
    assert torch.equal(counts, refs)
    assert not cache.free(refs, table, ints(held)).any()
    assert cache.device_error() == 0


def test_beams_of_codes_over_a_compaction():
    """The same in 8 bits without taking tokens back: results before and after a
    compaction agree to the bit."""
    from paper_2609_37988_gb300.serving import PagedCache
    g = gen(60)
    cache = PagedCache(n_layers=1, n_q_heads=10, n_kv_heads=2, head_dim=128, n_pages=64, page_size=16, bits=8)
    refs = torch.zeros(64, dtype=torch.int32, device="cuda")
    refs[::3] = 1  # pages of others
    none = torch.zeros((0, 9), dtype=torch.int32, device="cuda"), ints([])
    refs, table = cache.fork(refs, *none, ints([-1, -1]), ints([100, 70]))
    k, v = (randn(g, (170, 2, 128), BF16) for _ in range(2))
    cache.append(0, k, v, offsets([100, 70]), ints([100, 70]), table)
    refs, table = cache.fork(refs, table, ints([100, 70]), ints([1, 0, 1]), ints([71, 101, 71]))
    k, v, q = (randn(g, (3, h, 128), BF16) for h in (2, 2, 10))
    lens, cu = ints([71, 101, 71]), offsets([1, 1, 1])
    cache.append(0, k, v, cu, lens, table)
    a = cache.attend(0, q, cu, lens, table, 0.088, max_new=1)
    refs[::3] = 0  # the others let go
    refs2, table2, where = cache.compact(refs, table, lens)
    assert not torch.equal(table, table2)
    b = cache.attend(0, q, cu, lens, table2, 0.088, max_new=1)
    assert torch.equal(a, b) and cache.device_error() == 0


def test_fork_of_as_many_rows_as_there_may_be():
    page, R, B, width, n_pages = 16, 16384, 700, 5, 40000
    g = np.random.default_rng(78)
    lens = [int(g.integers(0, 4)) * page + (int(g.integers(1, page)) if b % 20 == 0 else 0) for b in range(B)]
    refs, table = table_of(g, n_pages, page, lens, width, shared=300)
    parents = [int(x) for x in g.integers(-1, B, R)]
    after = [(lens[p] if p >= 0 else 0) + int(g.integers(0, 2)) * page for p in parents]
    pool = Pool(n_pages, page, 8, layers=1, hkv=1)
    refs2, out, copies, short = paged.fork(refs, table, lens, parents, after, width, page)
    assert short == 0 and len(copies) > 500
    got_refs, got = pool.cache.fork(*[ints(x) for x in (refs.tolist(), table.tolist(), lens, parents, after)])
    np.testing.assert_array_equal(got.cpu().numpy(), out)
    np.testing.assert_array_equal(got_refs.cpu().numpy(), refs2)
    pool.moved(copies)
