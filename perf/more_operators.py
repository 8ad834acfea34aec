"""Cases, plain forms and exact values of the operators of streams whose window slides.

A pool of pages holds the latents of many rollouts that never end: each stream keeps its first tokens (the sinks, visible for good) and a window of its newest
ones, and gives back the pages between them. Four operators:
  attention  new tokens over the sinks and a window of their stream, token by token or block by block; the sinks may be scored by queries rotated for them
  slide      pages that lie between sinks and window are given back, and the streams' page lists close up
  plan       token counts of a step to the places of its rows and the lengths to resize to
  positions  the coordinates of a step's tokens, absolute and relative to the sinks, and their rows in the pool
A stream's token of index i (counted from its start) lies at place i while nothing was given back, and `dropped` places further ahead behind the sinks' pages
afterwards. A case's sizes are its own; the values in it come from the seed.
"""
import math

import torch

own = False

GOLD = 0.6180339887498949
HEAD_DIM = 128


# ---------------------------------------------------------------- cases
def _attn(name, seqs, new, ctx, window, sinks, block, page, heads=12, d_c=192, d_r=32, ragged=True, slid=True, turned=True):
    return {"name": name, "op": "attention", "seqs": seqs, "new": new, "ctx": ctx, "window": window, "sinks": sinks, "block": block, "page": page, "heads": heads,
            "d_c": d_c, "d_r": d_r, "ragged": ragged, "slid": slid, "turned": turned}


def _slide(name, seqs, held, keep, sinks, page):
    return {"name": name, "op": "slide", "seqs": seqs, "held": held, "keep": keep, "sinks": sinks, "page": page}


def _plan(name, seqs, new):
    return {"name": name, "op": "plan", "seqs": seqs, "new": new}


def _positions(name, seqs, new, ctx, window, sinks, block, page, frame, width, ragged=True):
    return {"name": name, "op": "positions", "seqs": seqs, "new": new, "ctx": ctx, "window": window, "sinks": sinks, "block": block, "page": page, "frame": frame,
            "width": width, "ragged": ragged, "slid": True}


def listed():
    return [
        # one stream, one new token over a short history: the latency of a call
        _attn("window 1 token", 1, 1, 777, 512, 4, 1, 16, ragged=False, slid=False, turned=False),
        # a decoding step of 64 rollouts: a sink frame of 1560 tokens, rotated for, and the newest six frames
        _attn("window decode x64", 64, 1, 32760, 9360, 1560, 1, 64),
        # four rollouts' three-frame chunks far into a long video, bidirectional inside the chunk, one sink frame and the newest six
        _attn("window chunk x4", 4, 4680, 46800, 9360, 1560, 4680, 64, ragged=False),
        # ragged prompts in small pages, causal token by token, a short window and four first tokens
        _attn("window ragged prompts", 9, 3333, 8000, 1024, 4, 1, 16, heads=16, d_c=128, d_r=64, slid=False, turned=False),
        # a few drafted tokens of each stream verified at once, widest latents, sinks that end inside a page
        _attn("window verify d_c 512", 16, 5, 30000, 4096, 100, 1, 32, heads=16, d_c=512, d_r=64),
        # one long prompt from its first token on
        _attn("window long prompt", 1, 28000, 28000, 4096, 16, 1, 128, heads=8, d_c=256, d_r=32, ragged=False, slid=False, turned=False),
        # 64 rollouts past their windows by up to a few chunks give their pages back
        _slide("slide x64", 64, 24000, 9360, 1560, 64),
        # a thousand streams in small pages
        _slide("slide x1024", 1024, 8192, 4096, 4, 16),
        # a step of 64 streams
        _plan("plan x64", 64, 5),
        # as many streams as a pool may have
        _plan("plan x65536", 65536, 9),
        # a decoding step of 64 rollouts on the grid of 30 x 52 tokens a frame
        _positions("positions x64", 64, 1, 32760, 9360, 1560, 1, 64, 1560, 52),
        # ragged chunks of 16 rollouts
        _positions("positions chunks", 16, 4680, 46800, 9360, 1560, 4680, 64, 1560, 52),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_attn(rng):
    while True:
        d_c, d_r = rng.choice((64, 128, 192, 192, 256, 512)), rng.choice((32, 64))
        heads, page = rng.choice((8, 12, 12, 16)), rng.choice((16, 32, 64, 64, 120, 128))
        if rng.random() < 0.5:  # decoding: a token or a few drafted ones of many streams
            seqs, new = _log(rng, 1, 96), rng.choice((1, 1, 2, 5))
        else:  # chunks and prompts of a few
            seqs, new = _log(rng, 1, 8), _log(rng, 17, 4680)
        ctx = _log(rng, max(new, 65), 65520)
        window, sinks = _log(rng, 16, 16384), rng.choice((0, 1, 4, 64, 333, 1560))
        c = _attn("", seqs, new, ctx, window, sinks, rng.choice((1, 1, 0, new)), page, heads, d_c, d_r, rng.random() < 0.7, rng.random() < 0.6, rng.random() < 0.5)
        rows, held = seqs * new * heads, max(_lens(c)[1])
        # no more than the largest listed case, in memory of the plain form and in work
        if rows * held <= 224640 * 10976 and rows * min(held, window + sinks) * (2 * d_c + d_r) <= 224640 * 10920 * 416 and seqs * held * (d_c + d_r) <= 64 * 10976 * 224:
            return c


def _draw_meta(rng):
    page = rng.choice((16, 32, 64, 120, 128))
    kind = rng.random()
    if kind < 0.4:
        seqs = _log(rng, 1, 1024)
        held = _log(rng, 64, 8192 * 1024 // seqs if seqs > 128 else 65536)
        return _slide("", seqs, held, _log(rng, 1, held), rng.choice((0, 1, 4, 64, 1560)), page)
    if kind < 0.6:
        return _plan("", _log(rng, 1, 65536), _log(rng, 1, 4680))
    seqs = _log(rng, 1, 64)
    new = _log(rng, 1, 74880 // seqs if seqs > 16 else 4680)
    frame, width = rng.choice(((1560, 52), (64, 8), (1, 1)))
    return _positions("", seqs, new, new + _log(rng, 1, 60000), _log(rng, 16, 16384), rng.choice((0, 4, 1560)), rng.choice((1, 0, new)), page, frame, width)


def draw(rng):
    c = rng.choice((_draw_attn, _draw_attn, _draw_meta))(rng)
    del c["name"]
    return c


# ---------------------------------------------------------------- sizes that follow from a case
def _front(case):
    """Places that hold the sinks' pages."""
    return -(-case["sinks"] // case["page"]) * case["page"]


def _lens(case):
    """(new tokens, tokens held after them, tokens given back) of every stream."""
    n, held, gone, p, front = [], [], [], case["page"], _front(case)
    for s in range(case["seqs"]):
        f, g = ((s + 1) * GOLD) % 1.0, ((s + 1) * GOLD * GOLD * 3) % 1.0
        if not case["ragged"] or s == 0:
            n.append(case["new"])
            ctx = case["ctx"]
        else:
            n.append(0 if s % 8 == 7 else max(1, math.ceil(case["new"] * f)))  # every eighth stream idles
            ctx = max(n[-1], math.ceil(case["ctx"] * g))
        # a server that gave back what the step's first token does not see any more
        back = max(0, (ctx - n[-1] - case["window"]) // p - front // p) * p if case["slid"] else 0
        held.append(ctx - back)
        gone.append(back)
    return n, held, gone


def _ends(case, n, held, gone):
    """Where the keys end that each of a stream's new tokens sees, as indices."""
    i = torch.arange(held + gone - n, held + gone)
    b = case["block"]
    return torch.full_like(i, held + gone) if b == 0 else ((i // b + 1) * b).clamp(max=held + gone)


def _slide_lens(case):
    return [max(1, math.ceil(case["held"] * (((s + 1) * GOLD) % 1.0))) for s in range(case["seqs"])]


def work(case):
    op = case["op"]
    if op == "attention":
        pairs = keys = rows = 0
        sinks, window, front = case["sinks"], case["window"], _front(case)
        for ns, ks, gs in zip(*_lens(case)):
            if not ns:
                continue
            end = _ends(case, ns, ks, gs)
            base = front + gs if gs else sinks  # index of the first key that is no sink
            low = (end - window).clamp(min=base)
            pairs += int((end.clamp(max=sinks) + (end - low).clamp(min=0)).sum())
            keys += min(sinks, int(end[-1])) + max(0, int(end[-1]) - int(low[0]))
            rows += ns * case["heads"]
        d_c, d_r = case["d_c"], case["d_r"]
        return {"bytes": 2 * (keys * (d_c + d_r) + rows * (2 * d_c + d_r * (2 if case["turned"] else 1))), "flops": 2 * pairs * case["heads"] * (2 * d_c + d_r)}
    if op == "slide":
        p, cells = case["page"], 0
        for s, k in enumerate(_slide_lens(case)):
            if s % 8 != 7:
                gone = max(0, (k - case["keep"]) // p - _front(case) // p)
                cells += 3 * gone + 2 * (-(-k // p) - _front(case) // p - gone) if gone else 0
        return {"bytes": 4 * cells + 20 * case["seqs"], "flops": 0}
    if op == "plan":
        return {"bytes": 20 * case["seqs"], "flops": 0}
    n, held, _ = _lens(case)
    t = sum(n)
    return {"bytes": 28 * t + 12 * case["seqs"] + 4 * sum(-(-m // case["page"]) for m in n), "flops": 0}


# ---------------------------------------------------------------- inputs
def _randn(g, shape, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(torch.bfloat16)


def _fill(g, shape):
    """Large bf16 buffers, drawn in pieces."""
    x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
    for part in x.view(-1).split(1 << 28):
        part.normal_(generator=g)
    return x


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(n):
    return torch.tensor([0] + n, dtype=torch.int32, device="cuda").cumsum(0, dtype=torch.int32)


def _table(lens, page, seed, spare=1):
    """Pages of streams of these lengths in random places of a pool: (table, pages of the pool)."""
    need = [-(-k // page) for k in lens]
    pages = sum(need) + max(2, sum(need) // 8)
    most = max(need) + spare
    place = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[: sum(need)].to(torch.int32)
    table = torch.full((len(lens), most), -1, dtype=torch.int32)
    table[torch.arange(most)[None] < torch.tensor(need)[:, None]] = place
    return table, pages


def _pool(case, lens, g, d_c, d_r):
    table, pages = _table(lens, case["page"], g.initial_seed())
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[table[table >= 0].long()] = 1
    return {"c": _fill(g, (1, pages, case["page"], d_c)), "kr": _fill(g, (1, pages, case["page"], d_r)), "table": table.cuda(), "lens": _ints(lens), "refs": refs.cuda()}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": dict(case), "front": _front(case) if "sinks" in case else 0}
    op = case["op"]
    if op == "attention":
        n, held, gone = _lens(case)
        st |= _pool(case, held, g, case["d_c"], case["d_r"])
        t, h, d_c, d_r = sum(n), case["heads"], case["d_c"], case["d_r"]
        st["dropped"], st["q_start"] = _ints(gone), _starts(n)
        st["q_c"] = _randn(g, (t, h, d_c), math.sqrt((HEAD_DIM - d_r) / d_c))
        # the same queries at two angles: two draws of the same distribution
        st["q_r"], st["q_sink"] = _randn(g, (t, h, d_r)), _randn(g, (t, h, d_r)) if case["turned"] else None
        st["o"] = torch.empty(t, h, d_c, dtype=torch.bfloat16, device="cuda")
        st["most"] = (max(n), max(held))
    elif op == "slide":
        lens = _slide_lens(case)
        table, pages = _table(lens, case["page"], seed)
        for s in range(3, len(lens), 4):  # every fourth stream is a branch that shares its parent's pages
            lens[s] = lens[s - 1]
            table[s] = table[s - 1]
        refs = torch.bincount(table[table >= 0].long(), minlength=pages).to(torch.int32)
        # the metadata in one buffer, so that a pass starts from one copy of it
        parts = [table.flatten(), torch.tensor(lens, dtype=torch.int32), refs, torch.randint(0, 99, (len(lens),), generator=torch.Generator().manual_seed(seed)) * case["page"]]
        flat = [torch.nn.functional.pad(x.to(torch.int32), (0, -x.numel() % 4)) for x in parts]
        st["before"] = torch.cat(flat).cuda()
        st["meta"] = st["before"].clone()
        views = [v[: x.numel()] for v, x in zip(st["meta"].split([x.numel() for x in flat]), parts)]
        st["table"], st["lens"], st["refs"], st["dropped"] = views[0].view(table.shape), views[1], views[2], views[3]
        st["keep"] = _ints([-1 if s % 8 == 7 else case["keep"] for s in range(len(lens))])
        # what the pages hold plays no part
        st["c"] = st["kr"] = torch.zeros(1, pages, case["page"], 8, dtype=torch.bfloat16, device="cuda")
    elif op == "plan":
        b = case["seqs"]
        n = torch.randint(0, case["new"] + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
        st["n_new"] = torch.where(torch.rand(b, generator=g, device="cuda") < 0.2, 0, n)  # a fifth idles
        st["lens"] = torch.randint(0, 60, (b,), generator=g, device="cuda", dtype=torch.int32) * 16
        st["dropped"] = torch.randint(0, 4, (b,), generator=g, device="cuda", dtype=torch.int32) * 16
        st["q_start"], st["new_lens"] = torch.empty(b + 1, dtype=torch.int32, device="cuda"), torch.empty(b, dtype=torch.int32, device="cuda")
        st["table"], st["refs"] = torch.full((b, 64), -1, dtype=torch.int32, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
        st["c"] = st["kr"] = torch.zeros(1, 64, 16, 8, dtype=torch.bfloat16, device="cuda")
    else:
        n, held, gone = _lens(case)
        st |= _pool(case, held, g, 8, 8)
        st["dropped"], st["q_start"], t = _ints(gone), _starts(n), sum(n)
        st["pos"], st["pos_sink"] = torch.empty(t, 3, dtype=torch.int32, device="cuda"), torch.empty(t, 3, dtype=torch.int32, device="cuda")
        st["rows"] = torch.empty(t, dtype=torch.int32, device="cuda")
    if own:
        from paper_2605_30351_gb300 import videomla as V
        st["cache"] = V.PagedCache(st["c"], st["kr"], st["table"], st["lens"], st["refs"])
        st["window"] = V.PagedWindow(case.get("window", 1), case.get("sinks", 0), st["dropped"])
        if op == "attention":
            st["workspace"] = torch.empty(V.mla_paged_workspace_bytes(st["cache"]), dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    op = st["case"]["op"]
    if op == "slide":
        st["meta"].copy_(st["before"])
    if own:
        return _run_own(st, op)
    return {"attention": _plain_attention, "slide": _plain_slide, "plan": _plain_plan, "positions": _plain_positions}[op](st)


def _run_own(st, op):
    from paper_2605_30351_gb300 import videomla as V
    case = st["case"]
    if op == "attention":
        V.mla_paged_window_attention(st["cache"], st["window"], 0, st["q_c"], st["q_r"], st["q_sink"], st["q_start"], HEAD_DIM, case["block"], st["workspace"], st["o"])
        return st["o"]
    if op == "slide":
        V.mla_pages_slide(st["cache"], st["window"], st["keep"])
        return st["table"], st["lens"], st["refs"], st["dropped"]
    if op == "plan":
        V.mla_paged_window_plan(st["cache"], st["window"], st["n_new"], st["q_start"], st["new_lens"])
        return st["q_start"], st["new_lens"], st["dropped"]
    V.mla_paged_window_positions(st["cache"], st["window"], st["q_start"], case["block"], case["frame"], case["width"], st["pos"], st["pos_sink"], st["rows"])
    return st["pos"], st["pos_sink"], st["rows"]


# ---------------------------------------------------------------- plain forms
def _owner(q_start, total):
    """(stream, place among the stream's new tokens) of every new token."""
    t = torch.arange(total, device=q_start.device)
    s = torch.searchsorted(q_start, t.to(torch.int32), right=True) - 1
    return s, t - q_start[s]


def _end_of(i, length, block):
    """Where the keys end that the token of index i sees, for streams of these lengths."""
    return length.expand_as(i) if block == 0 else torch.minimum(length, (i // block + 1) * block)


def _plain_attention(st):
    case, start = st["case"], st["q_start"].long()
    n, lens, gone = start[1:] - start[:-1], st["lens"].long(), st["dropped"].long()
    (new, held), p, h, d_c, sinks, front = st["most"], case["page"], case["heads"], case["d_c"], case["sinks"], st["front"]
    seqs, pages = lens.numel(), -(-held // p)
    at = st["table"][:, :pages].long().clamp(min=0)
    k = torch.cat((st["c"][0][at], st["kr"][0][at]), -1).float().view(seqs, pages * p, -1)
    i = torch.arange(new, device=k.device)
    rows = (start[:-1, None] + i).clamp(max=st["q_c"].shape[0] - 1)

    def queries(q_r):
        return torch.cat((st["q_c"], q_r), -1)[rows].float().view(seqs, new * h, -1)

    s = queries(st["q_r"]) @ k.transpose(1, 2)
    if st["q_sink"] is not None:
        s[:, :, :sinks] = queries(st["q_sink"]) @ k[:, :sinks].transpose(1, 2)
    j = torch.arange(pages * p, device=k.device)
    index = j + (j >= front) * gone[:, None]
    end = _end_of((lens + gone - n)[:, None] + i, (lens + gone)[:, None], case["block"])
    near = (index[:, None] >= (end - case["window"])[:, :, None]) & ((gone == 0)[:, None] | (j >= front))[:, None]
    sees = (near | (j < sinks)) & (index[:, None] < end[:, :, None]) & (j < lens[:, None])[:, None]
    s = s.mul_(1.0 / math.sqrt(HEAD_DIM)).view(seqs, new, h, -1).masked_fill_(~sees[:, :, None], -math.inf).view(seqs, new * h, -1)
    w = s.sub_(s.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    o = (w @ k[:, :, :d_c]) / w.sum(-1, keepdim=True).clamp(min=1e-30)
    s_of, i_of = _owner(st["q_start"], st["q_c"].shape[0])
    return o.view(seqs, new, h, d_c)[s_of, i_of].to(torch.bfloat16)


def _plain_slide(st):
    case, table, lens, refs, dropped, keep = st["case"], st["table"], st["lens"], st["refs"], st["dropped"], st["keep"]
    p, first = case["page"], st["front"] // case["page"]
    gone = torch.where(keep >= 0, ((lens - keep) // p - first).clamp(min=0), 0)[:, None]
    j = torch.arange(table.shape[1], device=table.device)
    out = (j >= first) & (j < first + gone)
    refs.scatter_add_(0, table.clamp(min=0).flatten().long(), -out.flatten().to(torch.int32))
    of = j + torch.where(j >= first, gone, 0)
    table.copy_(torch.where(of < table.shape[1], table.gather(1, of.clamp(max=table.shape[1] - 1).long()), -1))
    lens.sub_(gone[:, 0] * p)
    dropped.add_(gone[:, 0] * p)
    return table, lens, refs, dropped


def _plain_plan(st):
    n, lens = st["n_new"], st["lens"]
    st["q_start"][0] = 0
    st["q_start"][1:] = n.cumsum(0)
    st["new_lens"].copy_(torch.where(n > 0, lens + n, -1))
    st["dropped"].masked_fill_(lens == 0, 0)
    return st["q_start"], st["new_lens"], st["dropped"]


def _plain_positions(st):
    case, q_start = st["case"], st["q_start"]
    frame, width, p = case["frame"], case["width"], case["page"]
    s, i = _owner(q_start, st["rows"].numel())
    lens, gone = st["lens"].long()[s], st["dropped"].long()[s]
    place = lens - (q_start[s + 1] - q_start[s]) + i
    index = place + gone
    hidden = (_end_of(index, lens + gone, case["block"]) - case["window"] - case["sinks"]).clamp(min=0)
    t, rest = index // frame, index % frame
    st["pos"].copy_(torch.stack((t, rest // width, rest % width), 1))
    st["pos_sink"].copy_(torch.stack((t - hidden // frame, rest // width, rest % width), 1))
    st["rows"].copy_(st["table"][s, place // p].long() * p + place % p)
    return st["pos"], st["pos_sink"], st["rows"]


# ---------------------------------------------------------------- exact values
def exact(case, seed):
    if case["op"] != "attention":
        return None
    st = prepare(case, seed)
    p, d_c, sinks, front, out, row = case["page"], case["d_c"], case["sinks"], _front(case), [], 0
    for s, (ns, ks, gs) in enumerate(zip(*_lens(case))):
        if not ns:
            continue
        ids = st["table"][s, : -(-ks // p)].long()
        c = st["c"][0][ids].reshape(-1, d_c)[:ks].double()
        kr = st["kr"][0][ids].reshape(-1, case["d_r"])[:ks].double()
        place = torch.arange(ks, device="cuda")
        for a in range(0, ns, 512):  # a run of queries with the keys that one of them sees
            b = min(ns, a + 512)
            end = _ends(case, ns, ks, gs)[a:b].cuda()[:, None]
            is_sink = place < sinks
            index = torch.where(place < front, place, place + gs)
            seen = (index < end) & (is_sink | ((index >= end - case["window"]) & (place >= (front if gs else 0))))
            of = torch.nonzero(seen.any(0))[:, 0]
            v, k, hide, first = c[of], kr[of], ~seen[:, of], is_sink[of]
            for h in range(case["heads"]):
                q = slice(row + a, row + b)
                score = st["q_r"][q, h].double() @ k.T
                if st["q_sink"] is not None:
                    score = torch.where(first, st["q_sink"][q, h].double() @ k.T, score)
                score = (score + st["q_c"][q, h].double() @ v.T) / HEAD_DIM ** 0.5
                out.append((row + a, h, torch.softmax(score.masked_fill(hide, -math.inf), -1) @ v))
        row += ns
    o = torch.empty(row, case["heads"], d_c, dtype=torch.float64, device="cuda")
    for at, h, part in out:
        o[at : at + part.shape[0], h] = part
    return o
