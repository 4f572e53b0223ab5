"""Work of the serving operators: rotary positions, the paged cache's append
and attention, and attention over whole packed prompts.

Shapes are those of the repository's workloads: 14B-shaped layers (40 query /
8 KV heads of 128), 7B-shaped ones (28 / 4) and the head_dim-64 toy layer
(8 / 2).  Keys and values are N(0, 1) with a lognormal(0, 0.5) scale per (head,
channel), queries N(0, 1).  A batch's sequences are packed one behind another
in a flat token dimension (offsets ``cu``); ``ragged`` lengths lie between a
sixteenth of and all of the case's ``ctx`` (or ``new``).  Pages of the pool
are handed out in random order, and slots that hold no position hold other
numbers, as they do in a pool that was used before.

Four kinds of case:

* ``rotary``  the queries and keys of new tokens are rotated.
* ``append``  new tokens' keys (rotated on the way) and values enter the pages,
              their queries are rotated beside them.
* ``attend``  the last ``new`` tokens of each sequence attend over the pages.
* ``prompt``  whole prompts attend to themselves, causally.
"""
import math
import random

import torch

own = False

# (query heads, KV heads, head_dim)
MODELS = {"14b": (40, 8, 128), "7b": (28, 4, 128), "toy": (8, 2, 64)}
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BASE = 1000000.0


def listed():
    return [
        # one decode step's queries and keys of a 7B-shaped layer: latency
        _case("rotary", "7b", 16, 1, ctx=8192, name="rotary_step_7b"),
        # a video prompt, three axes (time, height, width)
        _case("rotary", "14b", 1, 16384, ctx=16384, axes=3, name="rotary_video_14b"),
        # a decode step's new tokens enter the pages
        _case("append", "14b", 32, 1, ctx=8192, page=16, name="append_step_14b"),
        # a batch of prompts of different lengths enters the pages
        _case("append", "7b", 9, 4001, ctx=4001, page=64, dtype="f16", ragged=True, axes=3, name="append_prompts_7b_f16"),
        # many short prompts of a small model in one call
        _case("prompt", "toy", 37, 301, ragged=True, name="prompt_toy_short"),
        # four prompts at the 14B shape, the length of its decode workload
        _case("prompt", "14b", 4, 8192, name="prompt_14b_8k"),
        # prompts of very different lengths at the 7B shape
        _case("prompt", "7b", 11, 9001, dtype="f16", ragged=True, name="prompt_7b_f16_ragged"),
        # a long prompt of a layer that looks back 4096 positions
        _case("prompt", "14b", 1, 32768, window=4096, name="prompt_14b_window"),
        # the smallest call: a single user's token over a short context
        _case("attend", "toy", 1, 1, ctx=512, page=16, name="attend_step_toy"),
        # a decode step at serving batch over the 14B workload's context
        _case("attend", "14b", 32, 1, ctx=8192, page=16, name="attend_step_14b"),
        # drafted tokens of a few users are checked, long odd contexts
        _case("attend", "7b", 7, 5, ctx=40001, page=32, dtype="f16", ragged=True, name="attend_draft_7b_f16"),
        # a chunk of long prompts over what is in the pages
        _case("attend", "14b", 4, 2048, ctx=32768, page=64, name="attend_chunk_14b"),
    ]


def _case(kind, model, batch, new, *, ctx=0, page=0, dtype="bf16", axes=1, window=0, ragged=False, pairs="half", part=1.0,
          name=None):
    c = dict(kind=kind, model=model, batch=batch, new=new, ctx=ctx or new, page=page, dtype=dtype, axes=axes,
             window=window, ragged=ragged, pairs=pairs, part=part)
    if name is not None:
        c["name"] = name
    return c


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi)))))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "prompt", "prompt", "prompt", "attend", "attend", "attend"])
    model = rng.choice(["14b", "14b", "7b", "7b", "toy"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    page = rng.choice([16, 32, 64, 128])
    ragged = rng.random() < 0.6
    if kind == "rotary":
        batch = _log(rng, 1, 64)
        return _case("rotary", model, batch, _log(rng, 1, 16384 // batch), ctx=131072, axes=rng.choice([1, 3, 3]),
                     dtype=rng.choice(["bf16", "f16", "f32"]), ragged=ragged, pairs=rng.choice(["half", "half", "adjacent"]),
                     part=rng.choice([1.0, 1.0, 0.5]))
    if kind == "append":
        batch = _log(rng, 1, 64)
        new = _log(rng, 1, 16384 // batch)
        return _case("append", model, batch, new, ctx=min(max(8192, new), 262144 // batch), page=page, dtype=dtype,
                     axes=rng.choice([1, 3]), ragged=ragged, pairs=rng.choice(["half", "half", "adjacent"]),
                     part=rng.choice([1.0, 1.0, 0.5]))
    if kind == "prompt":
        batch = _log(rng, 1, 64)
        return _case("prompt", model, batch, _log(rng, 64, 16384 // batch), dtype=dtype, ragged=ragged,
                     window=rng.choice([0, 0, 0, _log(rng, 16, 4096)]))
    batch = _log(rng, 1, 64)
    ctx = _log(rng, 128, min(65536, 262144 // batch))
    new = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, max(9, min(2048, 3500 // batch)))])
    return _case("attend", model, batch, min(new, ctx), ctx=ctx, page=page, dtype=dtype, ragged=ragged,
                 window=rng.choice([0, 0, 0, _log(rng, 64, 4096)]))


# -- inputs --------------------------------------------------------------------
def _lengths(case):
    """(new tokens, positions held with them) of every sequence, the same for every seed."""
    B, new, ctx = case["batch"], case["new"], case["ctx"]
    if not case["ragged"]:
        return [new] * B, [ctx] * B
    rng = random.Random(7919 * B + 31 * new + ctx)
    news = [_log(rng, max(1, new // 16), new) for _ in range(B)]
    if case["kind"] == "prompt":
        return news, news
    return news, [max(n, _log(rng, max(1, ctx // 16), ctx)) for n in news]


def _geometry(case):
    hq, hkv, d = MODELS[case["model"]]
    rot = int(d * case["part"])
    half = rot // 2
    if case["axes"] == 1:
        sections = [half]
    else:  # a quarter of the frequencies for time, three eighths each for height and width
        sections = [half // 4, half // 8 * 3, half - half // 4 - half // 8 * 3]
    return hq, hkv, d, rot, sections


def _positions(case, news, lens, dev):
    """Positions [axes, tokens]: of text on the first axis; a video's patches row by row on the others."""
    flat = torch.cat([torch.arange(l - n, l) for n, l in zip(news, lens)])
    if case["axes"] == 1:
        return flat.to(torch.int32).to(dev).unsqueeze(0)
    return torch.stack([flat // 256, flat // 16 % 16, flat % 16]).to(torch.int32).to(dev)


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    hq, hkv, d, rot, sections = _geometry(case)
    dt = DTYPES[case["dtype"]]
    news, lens = _lengths(case)
    n = sum(news)
    g = torch.Generator(device=dev).manual_seed(int(seed))
    scale_k = torch.exp(0.5 * torch.randn((hkv, d), generator=g, device=dev))
    scale_v = torch.exp(0.5 * torch.randn((hkv, d), generator=g, device=dev))
    s = dict(case=case, news=news, lens=lens, kind=case["kind"], sigma=d ** -0.5, window=case["window"])
    offs = [0]
    for x in news:
        offs.append(offs[-1] + x)
    s["offs"] = offs
    s["cu"] = torch.tensor(offs, dtype=torch.int32, device=dev)
    # the projection's output, of which q, k and v are views
    qkv = torch.randn((n, hq + 2 * hkv, d), generator=g, device=dev)
    qkv[:, hq: hq + hkv] *= scale_k
    qkv[:, hq + hkv:] *= scale_v
    qkv = qkv.to(dt)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq: hq + hkv], qkv[:, hq + hkv:]
    if s["kind"] in ("rotary", "append"):
        s["pos"] = _positions(case, news, lens, dev)
        axis = [a for a, m in enumerate(sections) for _ in range(m)]
        s["axis"] = torch.tensor(axis, device=dev)
        s["inv_freq"] = torch.tensor([BASE ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device=dev)
    if s["kind"] in ("append", "attend"):
        p = case["page"]
        per = [(l + p - 1) // p for l in lens]
        n_pages = sum(per) + 3
        order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
        table = torch.zeros((len(lens), max(per)), dtype=torch.int32)
        at = 0
        host = order.cpu()
        for b, m in enumerate(per):
            table[b, :m] = host[at: at + m]
            at += m
        s["table"] = table.to(dev)
        s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=dev)
        if s["kind"] == "attend":
            # [pages, KV heads, slots, channels]
            k = torch.empty((n_pages, hkv, p, d), dtype=dt, device=dev)
            v = torch.empty_like(k)
            for x, sc in ((k, scale_k), (v, scale_v)):
                for i in range(0, n_pages, 4096):
                    part = torch.randn(x[i: i + 4096].shape, generator=g, device=dev)
                    x[i: i + 4096] = (part * sc[:, None]).to(dt)
        else:
            k = torch.zeros((n_pages, hkv, p, d), dtype=dt, device=dev)
            v = torch.zeros_like(k)
        s["k_pages"], s["v_pages"] = k, v
    if own:
        from paper_2609_37988_gb300 import serving
        if s["kind"] in ("rotary", "append"):
            s["rotary"] = serving.Rotary(head_dim=d, rotary_dim=rot, base=BASE, sections=sections,
                                         adjacent=case["pairs"] == "adjacent")
        if s["kind"] in ("append", "attend"):
            s["cache"] = serving.PagedCache(n_q_heads=hq, k_pages=[s["k_pages"]], v_pages=[s["v_pages"]])
    return s


# -- the operators ---------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    kind = s["kind"]
    if kind == "rotary":
        c, n = _angles(s)
        return {"q": _rotate(s, s["q"], c, n), "k": _rotate(s, s["k"], c, n)}
    if kind == "append":
        c, n = _angles(s)
        q, k = _rotate(s, s["q"], c, n), _rotate(s, s["k"], c, n)
        page, slot = _places(s)
        s["k_pages"][page, :, slot] = k
        s["v_pages"][page, :, slot] = s["v"]
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=s["q"].device)
    for b, (n, l) in enumerate(zip(s["news"], s["lens"])):
        rows = slice(s["offs"][b], s["offs"][b + 1])
        if kind == "attend":
            p = s["case"]["page"]
            at = s["table"][b, : (l + p - 1) // p].long()
            hkv, d = s["k_pages"].shape[1], s["k_pages"].shape[3]
            k, v = (x[at].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :l].float() for x in (s["k_pages"], s["v_pages"]))
        else:
            k, v = (x[rows].permute(1, 0, 2).float() for x in (s["k"], s["v"]))
        out[rows] = _attend(s["q"][rows].float(), k, v, s["sigma"], s["window"]).to(out.dtype)
    return out


def _run_own(s):
    kind = s["kind"]
    if kind == "rotary":
        q, k = s["rotary"].apply(s["q"], s["k"], s["pos"])
        return {"q": q, "k": k}
    if kind == "append":
        q = s["cache"].append(0, s["k"], s["v"], s["cu"], s["lengths"], s["table"], rotary=s["rotary"], positions=s["pos"],
                              q=s["q"])
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if kind == "attend":
        return s["cache"].attend(0, s["q"], s["cu"], s["lengths"], s["table"], s["sigma"], max_new=max(s["news"]),
                                 window=s["window"])
    from paper_2609_37988_gb300 import serving
    return serving.prompt_attention(s["q"], s["k"], s["v"], s["cu"], s["sigma"], window=s["window"])


def _angles(s):
    """cos and sin [tokens, 1, frequencies]: angles in 64 bits, far positions lose theirs in 32."""
    a = s["pos"][s["axis"]].t().double() * s["inv_freq"]
    return torch.cos(a).float().unsqueeze(1), torch.sin(a).float().unsqueeze(1)


def _rotate(s, x, c, n):
    half = c.shape[-1]
    f = x.float()
    out = f.clone()
    if s["case"]["pairs"] == "half":
        a, b = f[..., :half], f[..., half: 2 * half]
        out[..., :half] = a * c - b * n
        out[..., half: 2 * half] = b * c + a * n
    else:
        a, b = f[..., 0: 2 * half: 2], f[..., 1: 2 * half: 2]
        out[..., 0: 2 * half: 2] = a * c - b * n
        out[..., 1: 2 * half: 2] = b * c + a * n
    return out.to(x.dtype)


def _places(s):
    """Page and slot of every packed token."""
    n = s["q"].shape[0]
    t = torch.arange(n, device=s["q"].device)
    b = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    pos = s["lengths"].long()[b] - s["cu"][1:].long()[b] + t
    p = s["case"]["page"]
    return s["table"].long()[b, pos // p], pos % p


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


# -- what the work is --------------------------------------------------------------
def _seen(n, l, window):
    """Positions that the last n of l queries see, all together."""
    w = window or l
    full = lambda m: m * (m + 1) // 2 if m <= w else w * (w + 1) // 2 + (m - w) * w  # noqa: E731
    return full(l) - full(l - n)


def work(case):
    hq, hkv, d, rot, _ = _geometry(case)
    e = 4 if case["dtype"] == "f32" else 2
    news, lens = _lengths(case)
    n = sum(news)
    if case["kind"] == "rotary":
        return {"bytes": 2 * n * (hq + hkv) * d * e + 4 * n * case["axes"], "flops": 3 * n * (hq + hkv) * rot}
    if case["kind"] == "append":
        return {"bytes": 2 * n * (hq + 2 * hkv) * d * e + 4 * n * (case["axes"] + 1), "flops": 3 * n * (hq + hkv) * rot}
    flops = sum(4 * d * hq * _seen(x, l, case["window"]) for x, l in zip(news, lens))
    w = case["window"]
    held = sum(min(l, x + w - 1) if w else l for x, l in zip(news, lens))
    return {"bytes": 2 * n * hq * d * e + 2 * held * hkv * d * e, "flops": flops}


def exact(case, seed):
    """From the definitions, in 64 bits: complex rotation, and attention one head at a time."""
    w = work(case)
    if case["kind"] in ("attend", "prompt") and w["flops"] > 1.2e13:
        return None
    s = prepare(case, seed)
    hq, hkv, d, rot, _ = _geometry(case)
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    if case["kind"] in ("rotary", "append"):
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=q.device),
                           s["pos"].double()[s["axis"]] * s["inv_freq"][:, None]).t()[:, None]

        def rotated(x):
            r = x[..., :rot]
            if case["pairs"] == "half":
                z = torch.complex(r[..., : rot // 2].contiguous(), r[..., rot // 2:].contiguous()) * turn
                y = torch.cat([z.real, z.imag], -1)
            else:
                y = torch.view_as_real(torch.view_as_complex(r.contiguous().unflatten(-1, (rot // 2, 2))) * turn).flatten(-2)
            return torch.cat([y, x[..., rot:]], -1)

        if case["kind"] == "rotary":
            return {"q": rotated(q), "k": rotated(k)}
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        kr, at, p = rotated(k), 0, case["page"]
        for b, (n, l) in enumerate(zip(s["news"], s["lens"])):
            where = torch.arange(l - n, l, device=q.device)
            pages, slots = s["table"][b].long()[where // p], where % p
            kp[pages, :, slots], vp[pages, :, slots] = kr[at: at + n], v[at: at + n]
            at += n
        return {"q": rotated(q), "k_pages": kp, "v_pages": vp}
    out = torch.empty((q.shape[0], hq, d), dtype=torch.float64, device=q.device)
    G, W, at = hq // hkv, case["window"], 0
    for b, (n, l) in enumerate(zip(s["news"], s["lens"])):
        if case["kind"] == "attend":
            where = torch.arange(l, device=q.device)
            pages, slots = s["table"][b].long()[where // case["page"]], where % case["page"]
        for h in range(hq):
            if case["kind"] == "attend":
                kk, vv = s["k_pages"][pages, h // G, slots].double(), s["v_pages"][pages, h // G, slots].double()
            else:
                kk, vv = k[at: at + n, h // G], v[at: at + n, h // G]
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
