"""Cases, plain forms and exact values of the paged-cache operators.

Four operators of a server that keeps many video streams' latents in one pool of pages:
  attention  a chunk of new tokens (or one token a stream) over the paged latent cache
  rope       rotary positions of part of a head, interleaved or half layout, forward or inverse
  append     new latents and rotated positional keys written into the streams' pages
  pages      fork streams and extend the branches (copy on write), or compact a fragmented pool
A case's sizes are its own; the values in it come from the seed.
"""
import math

import torch

own = False

GOLD = 0.6180339887498949
HEAD_DIM = 128


# ---------------------------------------------------------------- cases
def _attn(name, seqs, new, kv, block, page, heads=12, d_c=192, d_r=32, ragged=True):
    return {"name": name, "op": "attention", "seqs": seqs, "new": new, "kv": kv, "block": block, "page": page, "heads": heads, "d_c": d_c, "d_r": d_r,
            "ragged": ragged}


def _rope(name, tokens, heads, dim, rot, off, half, axes, dtype, inverse, context):
    return {"name": name, "op": "rope", "tokens": tokens, "heads": heads, "dim": dim, "rot": rot, "off": off, "half": half, "axes": axes, "dtype": dtype,
            "inverse": inverse, "context": context}


def _append(name, seqs, new, kv, page, d_c=192, d_r=32, ragged=True):
    return {"name": name, "op": "append", "seqs": seqs, "new": new, "kv": kv, "page": page, "d_c": d_c, "d_r": d_r, "ragged": ragged}


def _fork(name, layers, seqs, kv, new, page, d_c=192, d_r=32):
    return {"name": name, "op": "fork", "layers": layers, "seqs": seqs, "kv": kv, "new": new, "page": page, "d_c": d_c, "d_r": d_r}


def _compact(name, layers, pages, fill, row, page, d_c=192, d_r=32):
    return {"name": name, "op": "compact", "layers": layers, "pages": pages, "fill": fill, "row": row, "page": page, "d_c": d_c, "d_r": d_r}


def listed():
    return [
        # one stream, one new token over a short history: the latency of a call
        _attn("attention 1 token", 1, 1, 777, 1, 16, ragged=False),
        # a decoding step of 64 streams with up to a full 21-frame window of 1560 tokens each
        _attn("attention decode x64", 64, 1, 32760, 1, 64),
        # a three-frame chunk of the Wan layer against its full window, bidirectional inside the chunk
        _attn("attention chunk", 1, 4680, 32760, 4680, 64, ragged=False),
        # ragged prompts in small pages, causal token by token, narrow latents with wide positional keys
        _attn("attention ragged prompts", 9, 333, 5001, 1, 16, heads=16, d_c=128, d_r=64),
        # a few drafted tokens of each stream verified at once, widest latents
        _attn("attention verify d_c 512", 16, 5, 8190, 1, 32, heads=16, d_c=512, d_r=64),
        # positional queries of a decoding step
        _rope("rope step", 64, 12, 32, 32, 0, False, 3, "bfloat16", False, 1024),
        # queries of four chunks for dense attention: the last 32 of 128 channels turn
        _rope("rope chunk, part", 18720, 12, 128, 32, 96, False, 3, "bfloat16", False, 1024),
        # gradient of the half layout over a context stretched eight times, odd token count
        _rope("rope backward, long", 9999, 16, 128, 64, 0, True, 1, "float32", True, 131072),
        # the latents of one decoding step of 64 streams
        _append("append step", 64, 1, 4097, 64),
        # four streams' chunks
        _append("append chunks", 4, 4680, 32760, 64, ragged=False),
        # 12 rollouts branch and every branch grows by one chunk, all 30 layers
        _fork("fork and extend", 30, 12, 3001, 1560, 64),
        # a fragmented pool of 30 layers packed to its front
        _compact("compact pool", 30, 4096, 0.6, 74, 64),
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
        kv = _log(rng, max(new, 65), 32760)
        block = rng.choice((1, 1, 0, new))
        rows = seqs * new * heads
        if rows * kv <= 56160 * 32760 and rows * kv * (2 * d_c + d_r) <= 56160 * 32760 * 416 and seqs * kv * (d_c + d_r) <= 64 * 32760 * 224:
            return _attn("", seqs, new, kv, block, page, heads, d_c, d_r, rng.random() < 0.7)


def _draw_rope(rng):
    half, dim = rng.random() < 0.5, rng.choice((32, 64, 96, 128))
    rot = rng.choice([r for r in (16, 32, 64, 96, 128) if r <= dim])
    off = rng.choice((0, dim - rot))
    return _rope("", _log(rng, 3, 18720), rng.choice((1, 8, 12, 16)), dim, rot, off, half, 1 if half else rng.choice((1, 3)),
                 rng.choice(("bfloat16", "bfloat16", "float16", "float32")), rng.random() < 0.4, rng.choice((1024, 32768, 131072)))


def _draw_append(rng):
    seqs = _log(rng, 1, 64)
    new = _log(rng, 1, max(1, 18720 // seqs))
    return _append("", seqs, new, new + _log(rng, 1, 8000), rng.choice((16, 32, 64, 120, 128)), rng.choice((64, 128, 192, 256, 512)), rng.choice((32, 64)),
                   rng.random() < 0.5)


def _draw_pages(rng):
    layers, page = _log(rng, 1, 30), rng.choice((16, 32, 64, 128))
    if rng.random() < 0.5:
        return _fork("", layers, _log(rng, 1, 24), _log(rng, 40, 3001), _log(rng, 1, 1560), page)
    return _compact("", layers, _log(rng, 50, 4096 * 64 * 30 // (layers * page) if layers * page >= 960 else 8192), rng.choice((0.3, 0.6, 0.9)), _log(rng, 8, 200),
                    page)


def draw(rng):
    c = rng.choice((_draw_attn, _draw_attn, _draw_attn, _draw_rope, _draw_append, _draw_pages))(rng)
    del c["name"]
    return c


# ---------------------------------------------------------------- sizes that follow from a case
def _sizes(case):
    """(new tokens, tokens held after them) of every stream."""
    n, kv = [], []
    for s in range(case["seqs"]):
        f, g = ((s + 1) * GOLD) % 1.0, ((s + 1) * GOLD * GOLD * 3) % 1.0
        if not case["ragged"] or s == 0:
            n.append(case["new"])
            kv.append(case["kv"])
            continue
        n.append(0 if s % 8 == 7 else max(1, math.ceil(case["new"] * f)))  # every eighth stream idles
        kv.append(max(n[-1], math.ceil(case["kv"] * g)))
    return n, kv


def _visible(case, n, kv):
    """Pairs of a new token and a key that it sees, over all streams."""
    total, b = 0, case["block"]
    for ns, ks in zip(n, kv):
        a = torch.arange(ks - ns, ks)
        total += int((ks if b == 0 else torch.minimum(torch.tensor(ks), (a // max(b, 1) + 1) * b)).sum()) if b else ns * ks
    return total


def _fork_sizes(case):
    return [max(1, math.ceil(case["kv"] * (((s + 1) * GOLD) % 1.0))) for s in range(case["seqs"])]


def work(case):
    op = case["op"]
    if op == "attention":
        n, kv = _sizes(case)
        d_c, d_r, rows = case["d_c"], case["d_r"], sum(n) * case["heads"]
        held = sum(k for m, k in zip(n, kv) if m)
        return {"bytes": 2 * (held * (d_c + d_r) + rows * (2 * d_c + d_r)), "flops": 2 * _visible(case, n, kv) * case["heads"] * (2 * d_c + d_r)}
    if op == "rope":
        size = 4 if case["dtype"] == "float32" else 2
        values = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * size * values + 4 * case["tokens"] * (case["axes"] + case["rot"]), "flops": 3 * case["tokens"] * case["heads"] * case["rot"]}
    if op == "append":
        t = sum(_sizes(case)[0])
        return {"bytes": 4 * t * (case["d_c"] + case["d_r"]) + t * (12 + 4 * case["d_r"]), "flops": 3 * t * case["d_r"]}
    row = 2 * (case["d_c"] + case["d_r"]) * case["layers"]
    if op == "fork":
        lens, p = _fork_sizes(case), case["page"]
        cells = 2 * case["seqs"] * -(-(case["kv"] + case["new"]) // p)
        return {"bytes": 2 * row * sum(k % p for k in lens) + 8 * cells, "flops": 0}
    live, moved = _compact_sizes(case)
    return {"bytes": 2 * row * case["page"] * moved + 8 * (case["pages"] + live), "flops": 0}


def _compact_sizes(case):
    """(live pages, pages that have to move)."""
    live = max(1, int(case["pages"] * case["fill"]))
    return live, max(1, int((case["pages"] - live) * case["fill"]))


# ---------------------------------------------------------------- inputs
def _randn(g, shape, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _fill(g, shape):
    """Large bf16 buffers, drawn in pieces."""
    x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
    for part in x.view(-1).split(1 << 28):
        part.normal_(generator=g)
    return x


def _table(rot, context, theta=10000.0, native=1024):
    """cos and sin of every position, [context, rot / 2, 2]: past `native` positions the low frequencies are stretched (YaRN)."""
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    freq, size, s = theta ** (-2 * i / rot), 1.0, context / native
    if s > 1:
        turns = native * freq / (2 * math.pi)
        keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
        freq, size = freq / s * (1 - keep) + freq * keep, 0.1 * math.log(s) + 1
    a = torch.arange(context, dtype=torch.float64, device="cuda")[:, None] * freq
    return (torch.stack((a.cos(), a.sin()), -1) * size).float()


def _axes(pairs, axes):
    """Pairs that turn with each coordinate."""
    return (pairs - 2 * (pairs // 3), pairs // 3, pairs // 3) if axes == 3 else (pairs, 0, 0)


def _axis(pairs):
    return torch.repeat_interleave(torch.arange(3), torch.tensor(pairs)).cuda()


def _pool(case, g, lens, layers=1, extra=0):
    """Pages of streams of these lengths in random places of a pool, refs and table."""
    p = case["page"]
    need = [-(-k // p) for k in lens]
    pages = sum(need) + extra + max(2, sum(need) // 8)
    most = max(need) + 1
    place = torch.randperm(pages, generator=torch.Generator().manual_seed(g.initial_seed()))[: sum(need)].to(torch.int32)
    table = torch.full((len(lens), most), -1, dtype=torch.int32)
    table[torch.arange(most)[None] < torch.tensor(need)[:, None]] = place
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[place.long()] = 1
    return {"c": _fill(g, (layers, pages, p, case["d_c"])), "kr": _fill(g, (layers, pages, p, case["d_r"])), "table": table.cuda(),
            "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "refs": refs.cuda()}


def _cache(st):
    from paper_2605_30351_gb300 import videomla as V
    return V.PagedCache(st["c"], st["kr"], st["table"], st["lens"], st["refs"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": dict(case)}
    op = case["op"]
    if op == "attention":
        n, kv = _sizes(case)
        st |= _pool(case, g, kv)
        t, h, d_c, d_r = sum(n), case["heads"], case["d_c"], case["d_r"]
        st["q_start"] = torch.tensor([0] + n, dtype=torch.int32, device="cuda").cumsum(0, dtype=torch.int32)
        st["q_c"] = _randn(g, (t, h, d_c), std=math.sqrt((HEAD_DIM - d_r) / d_c))
        st["q_r"] = _randn(g, (t, h, d_r))
        st["o"] = torch.empty(t, h, d_c, dtype=torch.bfloat16, device="cuda")
        st["most"] = (max(n), max(kv))
        if own:
            from paper_2605_30351_gb300 import videomla as V
            st["cache"] = _cache(st)
            st["workspace"] = torch.empty(V.mla_paged_workspace_bytes(st["cache"]), dtype=torch.uint8, device="cuda")
    elif op == "rope":
        t, dtype = case["tokens"], getattr(torch, case["dtype"])
        st["x"] = _randn(g, (t, case["heads"], case["dim"]), dtype)
        st["y"] = torch.empty_like(st["x"])
        st["table"], st["axis"] = _table(case["rot"], case["context"]), _axis(_axes(case["rot"] // 2, case["axes"]))
        st["pos"] = torch.randint(0, case["context"], (t, case["axes"]), generator=g, device="cuda", dtype=torch.int32)
        if own:
            from paper_2605_30351_gb300 import videomla as V
            st["rope"] = V.Rope(st["table"], _axes(case["rot"] // 2, case["axes"]), offset=case["off"], half=case["half"])
    elif op == "append":
        n, kv = _sizes(case)
        st |= _pool(case, g, kv)
        t = sum(n)
        st["q_start"] = torch.tensor([0] + n, dtype=torch.int32, device="cuda").cumsum(0, dtype=torch.int32)
        st["c_new"], st["kr_new"] = _randn(g, (t, case["d_c"])), _randn(g, (t, case["d_r"]))
        st["rope_table"], st["axis"] = _table(case["d_r"], 1024), _axis(_axes(case["d_r"] // 2, 3))
        st["pos"] = torch.randint(0, 1024, (t, 3), generator=g, device="cuda", dtype=torch.int32)
        if own:
            from paper_2605_30351_gb300 import videomla as V
            st["cache"], st["rope"] = _cache(st), V.Rope(st["rope_table"], _axes(case["d_r"] // 2, 3))
    elif op == "fork":
        lens, p, b = _fork_sizes(case), case["page"], case["seqs"]
        new = sum(-(-(k + case["new"]) // p) - k // p for k in lens)
        st |= _pool(case, g, lens, case["layers"], extra=new)
        most = max(-(-(k + case["new"]) // p) for k in lens)
        table = torch.full((2 * b, most), -1, dtype=torch.int32, device="cuda")
        table[:b, : st["table"].shape[1]] = st["table"][:, :most]
        st["table"], st["lens"] = table, torch.cat((st["lens"], torch.zeros_like(st["lens"])))
        st["src"] = torch.arange(b, dtype=torch.int32, device="cuda")
        st["dst"] = st["src"] + b
        keep = torch.full_like(st["src"], -1)
        st["drop"] = torch.cat((keep, torch.zeros_like(keep)))
        st["grow"] = torch.cat((keep, st["lens"][:b] + case["new"]))
        if own:
            st["cache"] = _cache(st)
    else:
        live, moved = _compact_sizes(case)
        pages, row, p = case["pages"], case["row"], case["page"]
        host = torch.Generator().manual_seed(seed)
        front = torch.randperm(live, generator=host)[moved:]
        back = live + torch.randperm(pages - live, generator=host)[:moved]
        at = torch.cat((front, back))[torch.randperm(live, generator=host)].to(torch.int32)
        rows = -(-live // row)
        table = torch.full((rows + 1, row), -1, dtype=torch.int32)
        table.view(-1)[:live] = at
        table[rows] = table[0]  # a branch that shares the first stream's pages
        refs = torch.zeros(pages, dtype=torch.int32)
        refs[at.long()] = 1
        refs[table[0][table[0] >= 0].long()] = 2
        st |= {"c": _fill(g, (case["layers"], pages, p, case["d_c"])), "kr": _fill(g, (case["layers"], pages, p, case["d_r"])), "table": table.cuda(),
               "refs": refs.cuda(), "lens": ((table >= 0).sum(1) * p).to(torch.int32).cuda()}
        st["new_table"], st["new_refs"] = torch.empty_like(st["table"]), torch.empty_like(st["refs"])
        if own:
            st["cache"] = _cache(st)
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    op = st["case"]["op"]
    if own:
        return _run_own(st, op)
    return {"attention": _plain_attention, "rope": _plain_rope, "append": _plain_append, "fork": _plain_fork, "compact": _plain_compact}[op](st)


def _run_own(st, op):
    from paper_2605_30351_gb300 import videomla as V
    if op == "attention":
        V.mla_paged_attention(st["cache"], 0, st["q_c"], st["q_r"], st["q_start"], HEAD_DIM, st["case"]["block"], st["workspace"], st["o"])
        return st["o"]
    if op == "rope":
        V.mla_rope_apply(st["rope"], st["x"], st["pos"], st["y"], inverse=st["case"]["inverse"])
        return st["y"]
    if op == "append":
        V.mla_paged_append(st["cache"], 0, st["c_new"], st["kr_new"], st["q_start"], st["pos"], st["rope"])
        return st["c"].view(torch.int16), st["kr"]
    if op == "fork":
        V.mla_pages_resize(st["cache"], st["drop"])
        V.mla_pages_fork(st["cache"], st["src"], st["dst"])
        V.mla_pages_resize(st["cache"], st["grow"])
        return st["table"], st["lens"], st["refs"], st["c"].view(torch.int16), st["kr"].view(torch.int16)
    V.mla_pages_compact(st["cache"], st["new_table"], st["new_refs"])
    return st["new_table"], st["new_refs"], st["c"].view(torch.int16), st["kr"].view(torch.int16)


# ---------------------------------------------------------------- plain forms
def _owner(q_start, total):
    """(stream, place among the stream's new tokens) of every new token."""
    t = torch.arange(total, device=q_start.device)
    s = torch.searchsorted(q_start, t.to(torch.int32), right=True) - 1
    return s, t - q_start[s]


def _plain_attention(st):
    case, start = st["case"], st["q_start"].long()
    n, lens = start[1:] - start[:-1], st["lens"].long()
    (new, kv), p, h, d_c = st["most"], case["page"], case["heads"], case["d_c"]
    seqs, pages = lens.numel(), -(-kv // p)
    at = st["table"][:, :pages].long().clamp(min=0)
    k = torch.cat((st["c"][0][at], st["kr"][0][at]), -1).float().view(seqs, pages * p, -1)
    q = torch.cat((st["q_c"], st["q_r"]), -1)
    i = torch.arange(new, device=q.device)
    q = q[(start[:-1, None] + i).clamp(max=q.shape[0] - 1)].float().view(seqs, new * h, -1)
    here = lens[:, None] - n[:, None] + i  # each new token's place in its stream
    b = case["block"]
    sees = lens[:, None].expand(seqs, new) if b == 0 else torch.minimum(lens[:, None], (here // b + 1) * b)
    sees = torch.where(here >= 0, sees, 0).repeat_interleave(h, 1)
    j = torch.arange(pages * p, device=q.device)
    s = (q @ k.transpose(1, 2)).mul_(1.0 / math.sqrt(HEAD_DIM)).masked_fill_(j >= sees[:, :, None], -math.inf)
    w = s.sub_(s.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    v = k[:, :, :d_c] * (j < lens[:, None])[:, :, None]
    o = (w @ v) / w.sum(-1, keepdim=True).clamp(min=1e-30)
    s_of, i_of = _owner(st["q_start"], st["q_c"].shape[0])
    return o.view(seqs, new, h, d_c)[s_of, i_of].to(torch.bfloat16)


def _angles(table, pos, axis):
    """cos and sin of every token's pairs, [tokens, pairs]; pair i turns with coordinate axis[i]."""
    cs = table[pos.long()[:, axis], torch.arange(axis.numel(), device=pos.device)]
    return cs[..., 0], cs[..., 1]


def _turn(x, cos, sin, half):
    a, b = x.chunk(2, -1) if half else (x[..., 0::2], x[..., 1::2])
    y = (a * cos - b * sin, a * sin + b * cos)
    return torch.cat(y, -1) if half else torch.stack(y, -1).flatten(-2)


def _plain_rope(st):
    case, x = st["case"], st["x"].float()
    cos, sin = _angles(st["table"], st["pos"], st["axis"])
    a, b = case["off"], case["off"] + case["rot"]
    part = _turn(x[..., a:b], cos[:, None], -sin[:, None] if case["inverse"] else sin[:, None], case["half"])
    return torch.cat((x[..., :a], part, x[..., b:]), -1).to(st["x"].dtype)


def _slots(st):
    """The place in the pool of every new token."""
    p = st["case"]["page"]
    s, i = _owner(st["q_start"], st["c_new"].shape[0])
    at = st["lens"].long()[s] - (st["q_start"][s + 1] - st["q_start"][s]) + i
    return st["table"][s, at // p].long() * p + at % p


def _plain_append(st):
    cos, sin = _angles(st["rope_table"], st["pos"], st["axis"])
    slot = _slots(st)
    st["c"].view(-1, st["case"]["d_c"])[slot] = st["c_new"]
    st["kr"].view(-1, st["case"]["d_r"])[slot] = _turn(st["kr_new"].float(), cos, sin, False).to(torch.bfloat16)
    return st["c"].view(torch.int16), st["kr"]


def _plain_resize(st, new):
    """Streams take these lengths (-1: as it is): pages past the end are given back, then a shared last page that grows is copied and pages are added, the free
    page of the lowest number first, stream after stream."""
    p, table, refs = st["case"]["page"], st["table"], st["refs"]
    lens, new = st["lens"], torch.where(new < 0, st["lens"], new)
    have, want = -(-lens // p), -(-new // p)
    j = torch.arange(table.shape[1], device=table.device)
    gone = (j >= want[:, None]) & (j < have[:, None])
    refs.scatter_add_(0, table.clamp(min=0).flatten().long(), -gone.flatten().to(torch.int32))
    table.masked_fill_(gone, -1)
    last = table.gather(1, (have - 1).clamp(min=0)[:, None].long())[:, 0].clamp(min=0).long()
    copy = (new > lens) & (lens % p != 0) & (refs[last] > 1)
    need = (want - have).clamp(min=0) + copy
    begin = need.cumsum(0) - need
    free = torch.argsort((refs > 0).to(torch.int8), stable=True).to(torch.int32)
    at = begin[:, None] + copy[:, None] + j - have[:, None]
    added = (j >= have[:, None]) & (j < want[:, None])
    table.copy_(torch.where(added, free[at.clamp(0, free.numel() - 1)], table))
    to = torch.where(copy, free[begin.clamp(max=free.numel() - 1)].long(), last)
    held = torch.arange(p, device=table.device) < (lens % p)[:, None]
    for pool in (st["c"], st["kr"]):
        pool[:, to] = torch.where((held & copy[:, None])[None, :, :, None], pool[:, last], pool[:, to])
    table.copy_(torch.where(copy[:, None] & (j == have[:, None] - 1), to[:, None].to(torch.int32), table))
    taken = torch.arange(refs.numel(), device=refs.device) < need.sum()
    refs.scatter_add_(0, free.long(), taken.to(torch.int32))
    refs.scatter_add_(0, last, -copy.to(torch.int32))
    lens.copy_(new)


def _plain_fork(st):
    table, lens, refs, src, dst = st["table"], st["lens"], st["refs"], st["src"].long(), st["dst"].long()
    _plain_resize(st, st["drop"])
    rows = table[src]
    table[dst] = rows
    lens[dst] = lens[src]
    refs.scatter_add_(0, rows.clamp(min=0).flatten().long(), (rows >= 0).flatten().to(torch.int32))
    _plain_resize(st, st["grow"])
    return table, lens, refs, st["c"].view(torch.int16), st["kr"].view(torch.int16)


def _plain_compact(st):
    live = st["refs"] > 0
    i = torch.arange(live.numel(), device=live.device)
    front = i < live.sum()
    to, of = torch.nonzero(~live & front)[:, 0], torch.nonzero(live & ~front)[:, 0]
    where = i.to(torch.int32)
    where[of] = to.to(torch.int32)
    for pool in (st["c"], st["kr"]):
        pool[:, to] = pool[:, of]
    st["new_table"].copy_(torch.where(st["table"] >= 0, where[st["table"].clamp(min=0).long()], -1))
    st["new_refs"].copy_(torch.where(live & front, st["refs"], 0))
    st["new_refs"][to] = st["refs"][of]
    return st["new_table"], st["new_refs"], st["c"].view(torch.int16), st["kr"].view(torch.int16)


# ---------------------------------------------------------------- exact values
def _exact_attention(case, st):
    n, kv = _sizes(case)
    p, d_c, b, out, row = case["page"], case["d_c"], case["block"], [], 0
    for s, (ns, ks) in enumerate(zip(n, kv)):
        if not ns:
            continue
        ids = st["table"][s, : -(-ks // p)].long()
        c = st["c"][0][ids].reshape(-1, d_c)[:ks].double()
        k = st["kr"][0][ids].reshape(-1, case["d_r"])[:ks].double()
        a = torch.arange(ks - ns, ks, device="cuda")
        last = torch.full_like(a, ks) if b == 0 else (a.div(b, rounding_mode="floor") * b + b).clamp(max=ks)
        hidden = torch.arange(ks, device="cuda")[None] >= last[:, None]
        o = torch.empty(ns, case["heads"], d_c, dtype=torch.float64, device="cuda")
        for h in range(case["heads"]):
            score = st["q_c"][row : row + ns, h].double() @ c.T + st["q_r"][row : row + ns, h].double() @ k.T
            o[:, h] = torch.softmax((score / HEAD_DIM ** 0.5).masked_fill(hidden, -math.inf), -1) @ c
        out.append(o)
        row += ns
    return torch.cat(out)


def _exact_turn(x, pos, table, pairs, half, sign):
    x, y = x.double(), x.double().clone()
    m = sum(pairs)
    for i in range(m):
        axis = 0 if i < pairs[0] else 1 if i < pairs[0] + pairs[1] else 2
        cs = table[pos[:, axis].long(), i].double()
        z = torch.complex(cs[:, 0], sign * cs[:, 1])[:, None]
        u, v = (i, i + m) if half else (2 * i, 2 * i + 1)
        z = z * torch.complex(x[..., u], x[..., v])
        y[..., u], y[..., v] = z.real, z.imag
    return y


def exact(case, seed):
    op = case["op"]
    if op in ("fork", "compact"):
        return None
    st = prepare(case, seed)
    if op == "attention":
        return _exact_attention(case, st)
    if op == "rope":
        a, b = case["off"], case["off"] + case["rot"]
        y = st["x"].double()
        y[..., a:b] = _exact_turn(st["x"][..., a:b], st["pos"], st["table"], _axes(case["rot"] // 2, case["axes"]), case["half"], -1 if case["inverse"] else 1)
        return y
    turned = _exact_turn(st["kr_new"][:, None], st["pos"], st["rope_table"], _axes(case["d_r"] // 2, 3), False, 1)[:, 0]
    kr, p, row = st["kr"].double(), case["page"], 0
    for s, (ns, ks) in enumerate(zip(*_sizes(case))):
        a = torch.arange(ks - ns, ks, device="cuda")
        kr[0, st["table"][s, a // p].long(), a % p] = turned[row : row + ns]
        row += ns
    return None, kr
