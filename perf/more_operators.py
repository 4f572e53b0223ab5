"""Work of the paged cache in 8 bits and of the operators on pages.

Shapes are those of the repository's workloads: 14B-shaped layers (40 query / 8 KV
heads of 128), 7B-shaped ones (28 / 4) and the head_dim-64 toy layer (8 / 2).  Keys
and values are N(0, 1) with a lognormal(0, 0.5) scale per (head, channel), queries
N(0, 1).  New tokens are packed one behind another (offsets ``cu``); ``ragged``
lengths lie between a sixteenth of and all of the case's ``ctx`` (or ``new``).
Pages are handed out in random order, and slots that hold no position hold other
numbers, as they do in a pool that was used before.

A cache in 8 bits holds e4m3 codes and, for each page and KV head, an exponent of
its keys and one of its values: a number is code * 2^exponent.

Five kinds of case:

* ``append``   new tokens' keys and values enter the pages.
* ``attend``   the last ``new`` tokens of each sequence attend over the pages.
* ``copy``     pages are copied to other pages, in all layers.
* ``fork``     a batch's sequences go on from others (beams), or grow, are taken
               back, end and begin (a batch that is served); the pages that two
               would write to are copied, pages that nobody holds become free.
* ``compact``  a pool's used pages move to its beginning.
"""
import math
import random

import torch

own = False

# (query heads, KV heads, head_dim)
MODELS = {"14b": (40, 8, 128), "7b": (28, 4, 128), "toy": (8, 2, 64)}
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# exponents that a cache in 8 bits uses: its numbers are ones of the dtype
EXPS = {"bf16": (-110, 119), "f16": (-15, 7)}
E4M3 = torch.float8_e4m3fn


def listed():
    return [
        # a decode step's new tokens enter the pages
        _case("append", "14b", 32, 1, ctx=8192, page=16, name="append_step_14b"),
        # a batch of prompts of different lengths enters the pages
        _case("append", "7b", 9, 4001, ctx=4001, page=64, dtype="f16", ragged=True, name="append_prompts_7b_f16"),
        # the smallest call: a single user's token over a short context
        _case("attend", "toy", 1, 1, ctx=512, page=16, name="attend_step_toy"),
        # a decode step at serving batch over the 14B workload's context
        _case("attend", "14b", 32, 1, ctx=8192, page=16, name="attend_step_14b"),
        # drafted tokens of a few users are checked, long odd contexts
        _case("attend", "7b", 7, 5, ctx=40001, page=32, dtype="f16", ragged=True, name="attend_draft_7b_f16"),
        # a chunk of long prompts over what is in the pages
        _case("attend", "14b", 4, 2048, ctx=32768, page=64, name="attend_chunk_14b"),
        # one page of a small cache is copied: latency
        _pages("copy", "toy", 1, layers=2, n_pages=64, page=16, bits=8, name="copy_toy"),
        # a prefix of 4096 positions is doubled at the 14B shape, all its layers
        _pages("copy", "14b", 64, layers=48, n_pages=160, page=64, bits=16, name="copy_prefix_14b"),
        # beams of a batch of prompts go on from others, a token longer
        _pages("fork", "7b", 12, beams=8, layers=28, ctx=1501, page=16, bits=16, name="fork_beams_7b"),
        # a served batch between two steps: most sequences grow, some are taken back, end or begin
        _pages("fork", "14b", 256, layers=1, ctx=8192, page=16, bits=8, name="fork_served_14b"),
        # a small pool closes its gaps
        _pages("compact", "toy", 5, layers=2, n_pages=77, page=32, bits=8, name="compact_toy"),
        # a half empty pool closes its gaps, all layers
        _pages("compact", "7b", 40, layers=28, n_pages=2047, page=16, bits=16, name="compact_7b"),
    ]


def _case(kind, model, batch, new, *, ctx=0, page=16, dtype="bf16", window=0, ragged=False, name=None):
    c = dict(kind=kind, model=model, batch=batch, new=new, ctx=ctx or new, page=page, dtype=dtype, window=window, ragged=ragged)
    if name is not None:
        c["name"] = name
    return c


def _pages(kind, model, batch, *, layers, page, bits, beams=1, ctx=0, n_pages=0, name=None):
    """``batch``: pages to copy, prompts (times beams) or sequences."""
    c = dict(kind=kind, model=model, batch=batch, beams=beams, layers=layers, ctx=ctx, n_pages=n_pages, page=page, bits=bits,
             dtype="bf16")
    if name is not None:
        c["name"] = name
    return c


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "copy", "fork", "fork", "compact"])
    model = rng.choice(["14b", "14b", "7b", "7b", "toy"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    page = rng.choice([16, 32, 64, 128])
    ragged = rng.random() < 0.6
    if kind == "append":
        batch = _log(rng, 1, 64)
        new = rng.choice([1, _log(rng, 1, 16384 // batch)])
        return _case("append", model, batch, new, ctx=min(max(8192, new), 262144 // batch), page=page, dtype=dtype, ragged=ragged)
    if kind == "attend":
        batch = _log(rng, 1, 64)
        ctx = _log(rng, 128, min(65536, 262144 // batch))
        new = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, max(9, min(2048, 3500 // batch)))])
        return _case("attend", model, batch, min(new, ctx), ctx=ctx, page=page, dtype=dtype, ragged=ragged,
                     window=rng.choice([0, 0, 0, _log(rng, 64, 4096)]))
    # pools of 3 GB at most
    hq, hkv, d = MODELS[model]
    bits = rng.choice([8, 16])
    layers = 1 if model == "toy" else rng.choice([1, 4, 28])
    room = 3 * 2 ** 30 // (2 * layers * hkv * page * d * bits // 8)
    if kind == "copy":
        n_pages = _log(rng, 16, min(room, 20000))
        return _pages("copy", model, _log(rng, 1, n_pages // 3), layers=layers, n_pages=n_pages, page=page, bits=bits)
    if kind == "compact":
        n_pages = _log(rng, 16, min(room, 20000))
        return _pages("compact", model, _log(rng, 1, max(1, n_pages // 8)), layers=layers, n_pages=n_pages, page=page, bits=bits)
    beams = rng.choice([1, rng.randint(2, 10)])
    batch = _log(rng, 1, 256 // beams)
    ctx = _log(rng, 100, max(100, min(16384, room * page // (2 * batch) - 8 * page * beams)))
    if batch * (ctx // page + 8 * beams) > room:
        layers = 1
    return _pages("fork", model, batch, beams=beams, layers=layers, ctx=ctx, page=page, bits=bits)


# -- inputs --------------------------------------------------------------------
def _lengths(case):
    """(new tokens, positions held with them) of every sequence, the same for every seed."""
    B, new, ctx = case["batch"], case["new"], case["ctx"]
    if not case["ragged"]:
        return [new] * B, [ctx] * B
    rng = random.Random(7919 * B + 31 * new + ctx)
    news = [_log(rng, max(1, new // 16), new) for _ in range(B)]
    return news, [max(n, _log(rng, max(1, ctx // 16), ctx)) for n in news]


def _ceil(a, b):
    return (a + b - 1) // b


def _exponent(top, lo, hi):
    """Least e in [lo, hi] with top <= 448 * 2^e (448 = 0.875 * 2^9)."""
    m, e = torch.frexp(top)
    return torch.where(top > 0, e - 9 + (m > 0.875).int(), lo).clamp(lo, hi)


def _power(e):
    """2^e in binary32 (e within its normal exponents, else the nearest of them)."""
    return (e.int().clamp(-126, 127) + 127 << 23).view(torch.float32)


def _codes(x, e):
    """e4m3 codes (as bytes) of x over 2^e, rounded to nearest even."""
    y = (x * _power(-e.int())).clamp(-448, 448)
    return torch.where(x.isfinite(), y, math.nan).to(E4M3).view(torch.uint8)


def _values(codes, e):
    """What pages' codes (bytes) and exponents stand for, in binary32."""
    return codes.view(E4M3).float() * _power(e)[..., None, None]


def _fill(g, x, e, scale, dt, lim):
    """Pages x [n_pages, heads, slots, channels] of N(0, 1) * scale: numbers, or codes and exponents e."""
    step = max(1, 2 ** 27 // x[0].numel())
    for i in range(0, x.shape[0], step):
        part = torch.randn(x[i: i + step].shape, generator=g, device=x.device) * scale[:, None]
        part = part.to(dt)
        if e is not None:
            part = part.float()
            e[i: i + step] = _exponent(part.abs().amax((2, 3)), *lim).to(torch.int8)
            x[i: i + step].view(torch.uint8).copy_(_codes(part, e[i: i + step, :, None, None]))
        else:
            x[i: i + step] = part


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(int(seed))
    hq, hkv, d = MODELS[case["model"]]
    s = dict(case=case, kind=case["kind"], lim=EXPS[case["dtype"]])
    s["sk"] = torch.exp(0.5 * torch.randn((hkv, d), generator=g, device=dev))
    s["sv"] = torch.exp(0.5 * torch.randn((hkv, d), generator=g, device=dev))
    (_prepare_batch if s["kind"] in ("append", "attend") else _prepare_pages)(case, s, g, dev)
    if own:
        from paper_2609_37988_gb300 import serving
        s["cache"] = serving.PagedCache(n_q_heads=hq, k_pages=s["k_pages"], v_pages=s["v_pages"], k_exps=s["k_exps"],
                                        v_exps=s["v_exps"], dtype=DTYPES[case["dtype"]])
    return s


def _fill_pools(case, s, g, dev, n_pages, layers, held8):
    hq, hkv, d = MODELS[case["model"]]
    shape, s["out"] = (n_pages, hkv, case["page"], d), {}
    for name in "kv":  # all layers' pools in one allocation
        pages = torch.empty((layers,) + shape, dtype=E4M3 if held8 else DTYPES[case["dtype"]], device=dev)
        exps = torch.empty((layers,) + shape[:2], dtype=torch.int8, device=dev) if held8 else None
        for i in range(layers):
            _fill(g, pages[i], exps[i] if held8 else None, s["s" + name], DTYPES[case["dtype"]], s["lim"])
        s[name + "_pages"], s[name + "_exps"] = list(pages), list(exps) if held8 else None
        s["out"][name + "_pages"] = pages
        if held8:
            s["out"][name + "_exps"] = exps


def _prepare_batch(case, s, g, dev):
    hq, hkv, d = MODELS[case["model"]]
    dt, p = DTYPES[case["dtype"]], case["page"]
    news, lens = _lengths(case)
    n = sum(news)
    offs = [0]
    for x in news:
        offs.append(offs[-1] + x)
    s.update(news=news, lens=lens, offs=offs, sigma=d ** -0.5, window=case["window"])
    s["cu"] = torch.tensor(offs, dtype=torch.int32, device=dev)
    s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    # the projection's output, of which q, k and v are views
    qkv = torch.randn((n, hq + 2 * hkv, d), generator=g, device=dev)
    qkv[:, hq: hq + hkv] *= s["sk"]
    qkv[:, hq + hkv:] *= s["sv"]
    qkv = qkv.to(dt)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq: hq + hkv], qkv[:, hq + hkv:]
    per = [_ceil(l, p) for l in lens]
    n_pages = sum(per) + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32).cpu()
    table = torch.zeros((len(lens), max(per)), dtype=torch.int32)
    at = 0
    for b, m in enumerate(per):
        table[b, :m] = order[at: at + m]
        at += m
    s["table"] = table.to(dev)
    _fill_pools(case, s, g, dev, n_pages, 1, True)


def _prepare_pages(case, s, g, dev):
    """Pools of all layers; the pages' holders, the table and what is asked."""
    rng = random.Random(g.initial_seed())
    p, B = case["page"], case["batch"]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    if case["kind"] == "copy":
        n_pages = case["n_pages"]
        order = rng.sample(range(n_pages), 2 * B)
        s["src"], s["dst"] = ints(order[:B]), ints(order[B:])
    elif case["kind"] == "compact":
        # sequences over half of the pool's pages, anywhere in it; a quarter of them share their first pages with another
        n_pages = case["n_pages"]
        used = rng.sample(range(n_pages), max(B, n_pages // 2))
        shape = random.Random(7919 * B + n_pages)  # the lengths, the same for every seed
        cuts = sorted(shape.sample(range(1, len(used)), B - 1))
        rows = [used[a:b] for a, b in zip([0] + cuts, cuts + [len(used)])]
        for b in range(1, B, 4):
            rows[b] = rows[b - 1][: shape.randint(0, len(rows[b - 1]))] + rows[b]
        lens = [len(r) * p - shape.randint(0, p - 1) for r in rows]
        _state(s, rows, lens, n_pages, ints)
    else:
        # shared pages of every prompt, own ones of its beams behind them
        beams, ctx = case["beams"], case["ctx"]
        shape = random.Random(7919 * B + 31 * beams + ctx)  # the lengths, the same for every seed
        rows, lens, count = [], [], 0
        for _ in range(B):
            length = _log(shape, max(1, ctx // 16), ctx)
            shared = max(0, length // p - shape.randint(0, 3)) if beams > 1 else 0
            first = list(range(count, count + shared))
            count += shared
            for _ in range(beams):
                more = _ceil(length, p) - shared
                rows.append(first + list(range(count, count + more)))
                count += more
                lens.append(length)
        parents, after = [], []
        for i, length in enumerate(lens):
            if beams > 1:  # the prompt's best beams go on, some of them twice
                parents.append(i // beams * beams + rng.randrange(beams))
                after.append(length + 1)
            else:
                x = shape.random()  # the next token; a new prompt in its place; drafted tokens taken back; the end
                begins, back, ends = x < 0.04, 0.04 <= x < 0.10, 0.10 <= x < 0.12
                parents.append(-1 if begins or ends else i)
                after.append(_log(shape, 16, ctx) if begins else 0 if ends else max(0, length - shape.randint(1, 7)) if back
                             else length + 1)
        n_pages = count + sum(_ceil(a, p) - (0 if q < 0 else _ceil(lens[q], p)) + 1 for a, q in zip(after, parents)
                              if q < 0 or a > lens[q] or beams > 1) + 5
        order = list(range(n_pages))
        rng.shuffle(order)
        _state(s, [[order[x] for x in r] for r in rows], lens, n_pages, ints, spare=2)
        s["parents"], s["after"] = ints(parents), ints(after)
        width = max(_ceil(a, p) for a in after)
        if width > s["table"].shape[1]:
            s["table"] = torch.nn.functional.pad(s["table"], (0, width - s["table"].shape[1]), value=-1)
    _fill_pools(case, s, g, dev, n_pages, case["layers"], case["bits"] == 8)


def _state(s, rows, lens, n_pages, ints, spare=0):
    refs = [0] * n_pages
    for r in rows:
        for x in r:
            refs[x] += 1
    width = max(len(r) for r in rows) + spare
    s["refs"], s["lengths"] = ints(refs), ints(lens)
    s["table"] = ints([r + [-1] * (width - len(r)) for r in rows])


# -- the operators ---------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if own:
        cache = s["cache"]
        if kind == "append":
            cache.append(0, s["k"], s["v"], s["cu"], s["lengths"], s["table"])
            return s["out"]
        if kind == "attend":
            return cache.attend(0, s["q"], s["cu"], s["lengths"], s["table"], s["sigma"], max_new=max(s["news"]),
                                window=s["window"])
        if kind == "copy":
            cache.copy(s["src"], s["dst"])
            return s["out"]
        if kind == "fork":
            refs, table = cache.fork(s["refs"], s["table"], s["lengths"], s["parents"], s["after"])
            return dict(s["out"], refs=refs, table=table)
        refs, table, where = cache.compact(s["refs"], s["table"], s["lengths"])
        return dict(s["out"], refs=refs, table=table, where=where)
    if kind == "append":
        for new, pages, exps in ((s["k"], s["k_pages"][0], s["k_exps"][0]), (s["v"], s["v_pages"][0], s["v_exps"][0])):
            _append(s, new, pages.view(torch.uint8), exps)
        return s["out"]
    if kind == "attend":
        return _attend_pages(s)
    if kind == "copy":
        _copy(s, s["src"].long(), s["dst"].long())
        return s["out"]
    return (_fork if kind == "fork" else _compact)(s)


def _append(s, new, codes, exps):
    p, (lo, hi) = s["case"]["page"], s["lim"]
    n, dev = new.shape[0], new.device
    t = torch.arange(n, device=dev)
    b = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    first = s["lengths"].long()[b] - s["cu"].long()[b + 1] + s["cu"].long()[b]  # position of the sequence's first new token
    pos = first + t - s["cu"].long()[b]
    page, slot = s["table"].long()[b, pos // p], pos % p
    x = new.float()
    # per page: the largest magnitude that enters, and the slots filled before
    top = torch.zeros(exps.shape, device=dev)
    top.scatter_reduce_(0, page[:, None].expand(-1, exps.shape[1]), torch.where(x.isfinite(), x, 0).abs().amax(-1), "amax")
    filled = torch.zeros(exps.shape[0], dtype=torch.long, device=dev)
    filled[page] = (first - pos // p * p).clamp(min=0)
    at = torch.unique(page)
    old = exps[at].int()
    e = _exponent(top[at], lo, hi).int()
    e = torch.where(filled[at][:, None] > 0, torch.maximum(e, old), e)
    held = codes[at]
    again = _codes(held.view(E4M3).float(), (e - old)[..., None, None])
    before = torch.arange(p, device=dev) < filled[at][:, None]
    codes[at] = torch.where(before[:, None, :, None], again, held)
    exps[at] = e.to(torch.int8)
    codes[page, :, slot] = _codes(x, exps[page][..., None])


def _attend_pages(s):
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=s["q"].device)
    p = s["case"]["page"]
    pools = [(s["k_pages"][0].view(torch.uint8), s["k_exps"][0]), (s["v_pages"][0].view(torch.uint8), s["v_exps"][0])]
    for b, (n, l) in enumerate(zip(s["news"], s["lens"])):
        rows = slice(s["offs"][b], s["offs"][b + 1])
        at = s["table"][b, : _ceil(l, p)].long()
        k, v = (_values(x[at], e[at]).permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[3])[:, :l] for x, e in pools)
        out[rows] = _attend(s["q"][rows].float(), k, v, s["sigma"], s["window"]).to(out.dtype)
    return out


def _attend(q, k, v, sigma, window):
    """q [n, heads, d] at the last n of the positions of k, v [KV heads, t, d], 512 queries at a time."""
    n, hq, d = q.shape
    hkv, t, _ = k.shape
    out = torch.empty_like(q)
    for i in range(0, n, 512):
        x = q[i: i + 512]
        m = x.shape[0]
        first, last = t - n + i, t - n + i + m
        lo = max(0, first - window + 1) if window else 0
        x = x.reshape(m, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
        score = torch.bmm(x, k[:, lo:last].transpose(1, 2)).mul_(sigma).view(hkv, hq // hkv, m, last - lo)
        row = torch.arange(first, last, device=q.device)[:, None]
        col = torch.arange(lo, last, device=q.device)
        hidden = col > row
        if window:
            hidden |= col <= row - window
        score.masked_fill_(hidden, -math.inf)
        score -= score.amax(-1, keepdim=True)
        score.exp_()
        total = score.sum(-1, keepdim=True)
        y = torch.bmm(score.view(hkv, -1, last - lo), v[:, lo:last]).view(hkv, hq // hkv, m, d) / total
        out[i: i + 512] = y.permute(2, 0, 1, 3).reshape(m, hq, d)
    return out


def _copy(s, src, dst):
    for pages in s["k_pages"] + s["v_pages"]:
        x = pages.view(torch.uint8) if pages.dtype is E4M3 else pages
        x[dst] = x[src]
    for x in (s["k_exps"] or []) + (s["v_exps"] or []):
        x[dst] = x[src]


def _holders(table, count, n_pages):
    """How often each page stands in the first ``count`` entries of the table's rows."""
    col = torch.arange(table.shape[1], device=table.device)
    at = torch.where(col < count[:, None], table.long(), n_pages).flatten()
    return torch.zeros(n_pages + 1, dtype=torch.int32, device=table.device).index_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:-1]


def _fork(s):
    p, refs, table = s["case"]["page"], s["refs"], s["table"]
    n_pages, width, dev = refs.shape[0], table.shape[1], refs.device
    parent, after = s["parents"].long(), s["after"].long()
    held = s["lengths"].long()
    row = parent.clamp(min=0)
    kept = torch.minimum(torch.where(parent >= 0, held[row], 0), after)
    old, new, is_open = _ceil(kept, p), _ceil(after, p), kept % p != 0
    last = table.long()[row, (old - 1).clamp(min=0)]
    # a page that will be written to stays with the first that holds it so, if nobody else holds it
    same = parent[:, None] == parent
    whole = same & ((old > old[:, None]) | ((old == old[:, None]) & ~is_open))
    sooner = same & (old == old[:, None]) & is_open & (torch.arange(len(row), device=dev) < torch.arange(len(row), device=dev)[:, None])
    copied = is_open & ~((refs[last.clamp(0, n_pages - 1)] == 1) & ~whole.any(1) & ~sooner.any(1))
    need = copied.long() + new - old
    rank = need.cumsum(0) - need
    free = torch.argsort((refs != 0).to(torch.int8), stable=True)
    n_free = (refs == 0).sum()
    col = torch.arange(width, device=dev)
    fresh_from = (old - copied.long())[:, None]
    at = rank[:, None] + col - fresh_from
    fresh = torch.where(at < n_free, free[at.clamp(0, n_pages - 1)], -1)
    out = torch.where(col < fresh_from, table.long()[row], torch.where(col < new[:, None], fresh, -1)).to(torch.int32)
    counts = refs - _holders(table, _ceil(held, p), n_pages) + _holders(out, new, n_pages)
    pick = copied.nonzero().flatten()
    _copy(s, last[pick], out.long()[pick, old[pick] - 1])
    return dict(s["out"], refs=counts, table=out)


def _compact(s):
    p, refs, table = s["case"]["page"], s["refs"], s["table"]
    idx = torch.arange(refs.shape[0], device=refs.device)
    used = refs > 0
    low = idx < used.sum()
    src, dst = (used & ~low).nonzero().flatten(), (~used & low).nonzero().flatten()
    where = torch.where(used, idx, -1)
    where[src] = dst
    counts = torch.where(low, refs, 0)
    counts[dst] = refs[src]
    col = torch.arange(table.shape[1], device=refs.device)
    inside = col < _ceil(s["lengths"].long(), p)[:, None]
    out = torch.where(inside, where[table.long().clamp(min=0)], -1).to(torch.int32)
    _copy(s, src, dst)
    return dict(s["out"], refs=counts, table=out, where=where.to(torch.int32))


# -- what the work is --------------------------------------------------------------
def _seen(n, l, window):
    """Positions that the last n of l queries see, all together."""
    w = window or l
    full = lambda m: m * (m + 1) // 2 if m <= w else w * (w + 1) // 2 + (m - w) * w  # noqa: E731
    return full(l) - full(l - n)


def work(case):
    hq, hkv, d = MODELS[case["model"]]
    kind, p = case["kind"], case["page"]
    if kind in ("append", "attend"):
        news, lens = _lengths(case)
        n = sum(news)
        if kind == "append":
            return {"bytes": 2 * n * hkv * d * 3 + 8 * len(lens), "flops": 4 * n * hkv * d}
        w = case["window"]
        held = sum(min(l, x + w - 1) if w else l for x, l in zip(news, lens))
        return {"bytes": 2 * n * hq * d * 2 + 2 * held * hkv * d, "flops": sum(4 * d * hq * _seen(x, l, w) for x, l in zip(news, lens))}
    one = 2 * case["layers"] * hkv * p * d * case["bits"] // 8  # of a page, keys and values of all layers
    if kind == "copy":
        return {"bytes": case["batch"] * (2 * one + 8), "flops": case["batch"]}
    if kind == "compact":  # half of the pool is used, half of that lies behind where it will end
        n = case["n_pages"]
        return {"bytes": n // 4 * 2 * one + 12 * n + 4 * n, "flops": 4 * n}
    rows = case["batch"] * case["beams"]
    # a row's pages by the mean of its length's logarithm; of a prompt's beams (1 - 1/e) stand in a row, each keeping its page
    ctx = 0.34 * case["ctx"]
    table = 8 * rows * ctx / p
    copies = rows * 0.37 if case["beams"] > 1 else 0
    pages = rows * ctx / p if case["beams"] == 1 else case["batch"] * ctx / p + 2 * rows
    return {"bytes": int(copies * 2 * one + table + 8 * pages + 16 * rows), "flops": int(4 * pages + table / 2)}


def exact(case, seed):
    """From the definitions, in 64 bits: attention one head at a time, appended numbers over their page's power of two.
    What the operators on pages give are whole numbers and copies."""
    if case["kind"] not in ("append", "attend"):
        return None
    if case["kind"] == "attend" and work(case)["flops"] > 1.2e13:
        return None
    s = prepare(case, seed)
    hq, hkv, d = MODELS[case["model"]]
    p = case["page"]
    if case["kind"] == "append":
        out = {}
        for name in "kv":
            code, exps = s[name + "_pages"][0].double(), s[name + "_exps"][0]
            at = 0
            for b, (n, l) in enumerate(zip(s["news"], s["lens"])):
                for i in range((l - n) // p, _ceil(l, p)):
                    page = int(s["table"][b, i])
                    lo, hi = max(0, l - n - i * p), min(p, l - i * p)  # the new tokens' slots
                    x = s[name][at + i * p + lo - (l - n): at + i * p + hi - (l - n)].double().transpose(0, 1)
                    top = x.abs().flatten(1).amax(1).cpu()
                    for h in range(hkv):
                        e = s["lim"][0]
                        if float(top[h]) > 0:
                            e = min(s["lim"][1], max(e, math.ceil(math.log2(float(top[h]) / 448))))
                        if lo > 0:
                            e0 = int(exps[page, h])
                            e = max(e, e0)
                            code[page, h, :lo] *= 2.0 ** (e0 - e)
                        code[page, h, lo:hi] = x[h] * 2.0 ** -e
                at += n
            out[name + "_pages"] = code[None]
            out[name + "_exps"] = None
        return out
    k, v = ((s[x + "_pages"][0], s[x + "_exps"][0]) for x in "kv")
    q = s["q"].double()
    out = torch.empty((q.shape[0], hq, d), dtype=torch.float64, device=q.device)
    G, W, at = hq // hkv, case["window"], 0
    for b, (n, l) in enumerate(zip(s["news"], s["lens"])):
        where = torch.arange(l, device=q.device)
        pages, slots = s["table"][b].long()[where // p], where % p
        for h in range(hq):
            kk, vv = (torch.ldexp(x.view(torch.uint8)[pages, h // G, slots].view(E4M3).double(), e[pages, h // G].int()[:, None])
                      for x, e in (k, v))
            for i in range(0, n, 2048):
                rows = q[at + i: at + min(n, i + 2048), h]
                p0 = l - n + i
                p1 = p0 + rows.shape[0]
                c0 = max(0, p0 + 1 - W) if W else 0
                x = (rows @ kk[c0:p1].T) * d ** -0.5
                back = torch.arange(p0, p1, device=q.device)[:, None] - torch.arange(c0, p1, device=q.device)
                x = x.masked_fill((back < 0) | (back >= (W or l)), -math.inf)
                out[at + i: at + i + rows.shape[0], h] = torch.softmax(x, -1) @ vv[c0:p1]
        at += n
    return out
