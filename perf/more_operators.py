"""Rotary positions and a paged cache of 16-bit keys and values: operators whose speed is measured, with their plain forms.

A step over such a cache turns the new tokens' queries, puts their keys (turned on the way) and values into pages and attends over
the pages:

  table   (cos, sin) of positions times frequencies, angles in 64 bits, one position axis or several
  rope    rows turned by a table's rows, or their gradients turned back
  append  keys and values of new tokens into the sequences' pages
  attend  attention of the new tokens over the pages

A plain form is the operator's definition in elementary operations.  Sizes are those of
paper_2602_02958_amd/configs.py (heads, chunks as pages, cached tokens), or generic.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _case(name, op, defaults, kw):
    c = dict(op=op, **defaults)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def _table(name, **kw):
    """(cos, sin) of `tokens` positions and `pairs` frequencies.  axes: 1: places 0, 1, ..; 3: (frame, row, column) of a video's
    tokens.  scale: long contexts, the frequencies' factor by bands."""
    return _case(name, "table", dict(tokens=4096, pairs=64, axes=1, type="f16", scale=1), kw)


def _rope(name, **kw):
    """`seqs` x `heads` x `nodes` rows of `dim` channels, the first 2 * `pairs` turned.  half: pairs (i, i + pairs), else (2i, 2i + 1).
    given: a position for every token (anywhere in the table), else the sequence's first one.  backward: gradients."""
    return _case(name, "rope", dict(seqs=1, heads=12, nodes=1, dim=128, pairs=64, places=32768, type="bf16", table="f16", half=False,
                                    given=False, backward=False), kw)


def _append(name, **kw):
    """Up to `nodes` new tokens of `seqs` sequences behind up to `tokens` cached ones, pages of `page`; pairs 0: keys are not turned."""
    return _case(name, "append", dict(seqs=1, heads=12, nodes=1, tokens=4096, page=64, dim=128, pairs=64, type="bf16", table="f16", half=False,
                                      ragged=False), kw)


def _attend(name, **kw):
    """`nodes` new tokens of `seqs` sequences, `group` query heads to each of `heads` KV heads, over up to `tokens` tokens in pages (the new
    ones among them).  window > 0: the newest tokens that a row sees, beside the first `sink`."""
    return _case(name, "attend", dict(seqs=1, heads=12, group=1, nodes=1, tokens=4096, page=64, dim=128, type="bf16", causal=True, window=0, sink=0,
                                      lse=False, ragged=False), kw)


def listed():
    return [
        # the window's table, once a rollout
        _table("table_window", tokens=37440),
        # the longest rollout's, three axes, long contexts, 32 bits
        _table("table_long_axes", tokens=748800, axes=3, type="f32", scale=8),
        # one new token's queries: latency
        _rope("rope_token", heads=12, nodes=1),
        # a chunk's queries of a large model's layer
        _rope("rope_chunk", heads=40, nodes=10800, given=True),
        # gradients in 32 bits, odd sizes, a part of the head, the other pairing
        _rope("rope_back", seqs=3, heads=8, nodes=2049, dim=96, pairs=32, type="f32", table="f32", half=True, backward=True),
        # a decoding step of a batch, small pages
        _append("append_token", seqs=64, heads=8, tokens=511, page=16, half=True, ragged=True),
        # a chunk of 4680 tokens behind seven others
        _append("append_chunk", heads=12, nodes=4680, tokens=32760, page=4680),
        # ragged prompts, pages that end anywhere, a part of the head, binary16
        _append("append_prompts", seqs=7, heads=8, nodes=777, tokens=1500, page=100, dim=64, pairs=16, type="f16", table="f32", ragged=True),
        # one token of one head over a short cache: launches and latency
        _attend("attend_token", heads=1, tokens=1000, page=16),
        # a serving batch, four query heads to a KV head, ragged lengths
        _attend("attend_batch", seqs=16, heads=8, group=4, tokens=32768, page=64, ragged=True),
        # a few new tokens of a batch within a window and the first tokens, odd pages, binary16
        _attend("attend_window", seqs=5, heads=8, group=8, nodes=5, tokens=20000, page=100, dim=64, type="f16", window=4096, sink=40, lse=True,
                ragged=True),
        # one token over one layer of the longest rollout, chunks as pages
        _attend("attend_long_layer", tokens=748800, page=4680, lse=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["table", "rope", "rope", "append", "append"] + ["attend"] * 5)
    if op == "table":
        tokens = _log_int(rng, 1, 748800)
        return _table(None, tokens=tokens, pairs=rng.choice([8, 16, 30, 32, 48, 64, rng.randint(4, 64)]), axes=rng.choice([1, 3]),
                      type=rng.choice(["f16", "f32"]), scale=rng.choice([1, 1, 4, 8]))
    dim = rng.choice([64, 96, 128, 128, 128, 192, 256])
    pairs = rng.choice([dim // 2, dim // 2, dim // 4, 8 * rng.randint(1, dim // 16), rng.randint(4, dim // 2)])
    turn = dict(dim=dim, pairs=pairs, table=rng.choice(["f16", "f32"]), half=rng.random() < 0.5)
    if op == "rope":
        seqs, heads = _log_int(rng, 1, 32), _log_int(rng, 1, 64)
        nodes = _log_int(rng, 1, max(1, min(10800, 27_000_000 // (seqs * heads * dim))))
        return _rope(None, seqs=seqs, heads=heads, nodes=nodes, type=rng.choice(["bf16", "bf16", "f16", "f32"]), given=rng.random() < 0.5,
                     backward=rng.random() < 0.3, places=max(nodes, _log_int(rng, 64, 65536)), **turn)
    kind = rng.choice(["bf16", "bf16", "f16"])
    page = rng.choice([16, 32, 64, 128, _log_int(rng, 8, 4680), 8 * _log_int(rng, 2, 4680 // 8)])
    if op == "append":
        seqs, heads = _log_int(rng, 1, 64), _log_int(rng, 1, 40)
        most = max(2, 57_000_000 // (seqs * heads * dim))                   # tokens of a sequence
        nodes = rng.choice([1, _log_int(rng, 1, max(1, min(4680, most // 8)))])
        tokens = _log_int(rng, 1, max(1, min(32760, most - nodes)))
        page = min(page, max(8, most - nodes))
        if rng.random() < 0.2:
            turn["pairs"] = 0
        return _append(None, seqs=seqs, heads=heads, nodes=nodes, tokens=tokens, page=page, type=kind, ragged=seqs > 1 and rng.random() < 0.7,
                       **turn)
    heads, seqs = _log_int(rng, 1, 40), _log_int(rng, 1, 64)
    group = rng.choice([1, 1, 2, 4, 7, 8, 16])
    nodes = rng.choice([1, 1, 1, _log_int(rng, 2, 32)])
    most = min(748800, 12 * 748800 * 128 // (heads * seqs * dim), 1_500_000_000 // (heads * group * seqs * nodes))
    tokens = _log_int(rng, min(nodes + 1, most), most)
    window = rng.choice([0, 0, _log_int(rng, 1, 32768)])
    return _attend(None, seqs=seqs, heads=heads, group=group, nodes=nodes, tokens=tokens, page=page, dim=dim, type=kind,
                   causal=rng.random() < 0.8, window=window, sink=rng.choice([0, 4, 64, 1000]) if window else 0, lse=rng.random() < 0.5,
                   ragged=seqs > 1 and rng.random() < 0.7)


# ------------------------------------------------------------------------------------- inputs
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((seed * 1009 + what) % (1 << 62))


def _spread(c, most, what, low):
    """Lengths of the sequences, known from the case alone: all `most`, or spread over low..most with both ends among them."""
    n = c["seqs"]
    if not c["ragged"] or n == 1:
        return [most] * n
    out = [low + ((i * 7919 + what * 104729 + 31 * most) % 1000) * (most - low) // 1000 for i in range(n)]
    out[0], out[n - 1] = most, low
    return out


def _sizes(c):
    """Tokens in the cache (of an attention with the new ones, of an append without) and new ones of each sequence."""
    new = _spread(c, c["nodes"], 3, 1)
    kv = _spread(c, c["tokens"], 1, 1 if c["op"] == "attend" else 0)
    return ([max(a, b) for a, b in zip(kv, new)] if c["op"] == "attend" else kv), new


def _frequencies(pairs, scale):
    """Frequencies of base 10000; scale > 1: those of less than one turn in 4096 places slowed down by it, those of more than 32 not."""
    f = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64, device=DEV) / pairs)
    keep = ((f * 4096 / (2 * math.pi) - 1) / 31).clamp(0, 1)
    return f * (keep + (1 - keep) / scale)


def _axis(pairs):
    """The axis of each pair: the first pairs of a head go by the frame, then rows, then columns."""
    third = pairs // 3
    return [0] * (pairs - 2 * third) + [1] * third + [2] * third


def _rotary(c, places):
    """A table that the program keeps."""
    f = _frequencies(c["pairs"], 1)
    ang = torch.arange(places, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.stack([ang.cos(), ang.sin()], -1).to(TYPES[c["table"]]).contiguous()


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _pages(c, seed, lengths):
    """A pool that holds the lengths and one page more, each sequence's pages anywhere in it: (K and V pages [2, H, P, L, d], table).
    Behind a sequence's last page a table holds -1."""
    H, L, d = c["heads"], c["page"], c["dim"]
    used = [-(-n // L) for n in lengths]
    P = sum(used) + 1
    pool = torch.empty((2, H, P, L, d), dtype=TYPES[c["type"]], device=DEV)
    g = _gen(seed, 1)
    for side in pool:
        for unit in side:
            unit.copy_(torch.randn(unit.shape, generator=g, device=DEV))
    free = torch.randperm(P, generator=g, device=DEV).tolist()
    table = [[free.pop() for _ in range(u)] + [-1] * (max(used) - u) for u in used]
    return pool, _int32(table)


def prepare(case, seed):
    c, g = case, _gen(seed, 3)
    if c["op"] == "table":
        s = dict(case=c, freq=_frequencies(c["pairs"], c["scale"]), positions=None, axis=None)
        if c["axes"] == 3:
            # frames of 30 x 52 tokens, the first frame anywhere
            i = torch.arange(c["tokens"], device=DEV) + 1560 * int(torch.randint(0, 100, (1,), generator=g, device=DEV))
            s["positions"] = torch.stack([i // 1560, i // 52 % 30, i % 52], 1).to(torch.int32).contiguous()
            s["axis"] = _axis(c["pairs"])
        else:
            s["first"] = int(torch.randint(0, 1000, (1,), generator=g, device=DEV))
        return s
    kind = TYPES[c["type"]]

    def rows(heads):
        """[sequence, token, head, channel], as a projection leaves it, seen as [sequence, head, token, channel]."""
        return torch.randn((c["seqs"], c["nodes"], heads, c["dim"]), generator=g, device=DEV).to(kind).transpose(1, 2)

    if c["op"] == "rope":
        s = dict(case=c, x=rows(c["heads"]), table=_rotary(c, c["places"]), positions=None, first=None)
        if c["given"]:
            s["positions"] = torch.randint(0, c["places"], (c["seqs"], c["nodes"]), generator=g, device=DEV).to(torch.int32)
        else:
            s["first"] = torch.randint(0, c["places"] - c["nodes"] + 1, (c["seqs"],), generator=g, device=DEV).to(torch.int32)
        return s
    kv, new = _sizes(c)
    if c["op"] == "append":
        pool, table = _pages(c, seed, [a + b for a, b in zip(kv, new)])
        return dict(case=c, k=rows(c["heads"]), v=rows(c["heads"]), pool=pool, table=table, kv_len=_int32(kv), new=_int32(new),
                    rotary=_rotary(c, max(a + b for a, b in zip(kv, new))) if c["pairs"] else None)
    pool, table = _pages(c, seed, kv)
    return dict(case=c, q=rows(c["heads"] * c["group"]), pool=pool, table=table, kv_len=_int32(kv), new=_int32(new))


# ------------------------------------------------------------------------------- plain forms
def _plain_table(s):
    c = s["case"]
    if s["positions"] is None:
        pos = (s["first"] + torch.arange(c["tokens"], device=DEV))[:, None]
    else:
        pos = s["positions"][:, torch.tensor(s["axis"], device=DEV)]
    ang = pos.double() * s["freq"]
    return torch.stack([torch.cos(ang), torch.sin(ang)], -1).to(TYPES[c["type"]])


def _plain_turn(x, cs, half, backward=False):
    """Rows [B, H, N, d] in 32 bits by (cos, sin) [B, N, pairs, 2]."""
    p = cs.shape[2]
    cos, sin = cs.float()[:, None].unbind(-1)
    if backward:
        sin = -sin
    part, rest = x[..., :2 * p], x[..., 2 * p:]
    a, b = (part[..., :p], part[..., p:]) if half else (part[..., 0::2], part[..., 1::2])
    y = a * cos - b * sin, a * sin + b * cos
    y = torch.cat(y, -1) if half else torch.stack(y, -1).flatten(-2)
    return torch.cat([y, rest], -1)


def _plain_rope(s):
    c = s["case"]
    at = s["positions"] if s["positions"] is not None else s["first"][:, None] + torch.arange(c["nodes"], device=DEV)
    return _plain_turn(s["x"].float(), s["table"][at.long()], c["half"], c["backward"]).to(s["x"].dtype)


def _plain_append(s):
    c, L = s["case"], s["case"]["page"]
    k, v = s["k"].float(), s["v"]
    i = torch.arange(c["nodes"], device=DEV)
    at = s["kv_len"].long()[:, None] + i
    if s["rotary"] is not None:
        k = _plain_turn(k, s["rotary"][at.clamp(max=s["rotary"].shape[0] - 1)], c["half"])
    # a token behind the last one writes what the last one does
    j = torch.minimum(i[None], s["new"].long()[:, None] - 1)
    at = s["kv_len"].long()[:, None] + j
    page, row = s["table"].long().gather(1, at // L), at % L
    pick = j[:, None, :, None].expand(-1, c["heads"], -1, c["dim"])
    for side, x in zip(s["pool"], (k.to(v.dtype), v)):
        side[:, page, row] = x.gather(2, pick).transpose(0, 1)
    return s["pool"][0], s["pool"][1], s["kv_len"] + s["new"]


def _plain_attend(s):
    c = s["case"]
    n, H, G, m, L, d = c["seqs"], c["heads"], c["group"], c["nodes"], c["page"], c["dim"]
    K, V = (side[:, s["table"].long().clamp(min=0)].flatten(2, 3).transpose(0, 1).float() for side in s["pool"])       # [n, H, tokens, d]
    kv, new = s["kv_len"].long()[:, None, None], s["new"].long()[:, None, None]
    i, t = torch.arange(m, device=DEV)[None, :, None], torch.arange(K.shape[2], device=DEV)[None, None]
    place = kv - new + i
    see = (t < kv) & (i < new)
    if c["causal"]:
        see = see & (t <= place)
    if c["window"]:
        see = see & ((t > place - c["window"]) | (t < c["sink"]))
    x = torch.matmul(s["q"].float().reshape(n, H, G * m, d), K.transpose(2, 3)) * (1.0 / math.sqrt(d))
    x = torch.where(see[:, None, None], x.reshape(n, H, G, m, -1), -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(n, H, G * m, -1), V).reshape(n, H, G, m, d) / total.clamp(min=1e-38)
    o = o.reshape(n, H * G, m, d).to(s["q"].dtype)
    return (o, (top + torch.log(total)).reshape(n, H * G, m)) if c["lse"] else o


# ---------------------------------------------------------------------------------------- run
def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2602_02958_amd import binding as B
        if c["op"] == "table":
            if s["positions"] is None:
                return B.rope_table(c["tokens"], s["freq"], first=s["first"], dtype=TYPES[c["type"]])
            return B.rope_table(c["tokens"], s["freq"], positions=s["positions"], axis=s["axis"], dtype=TYPES[c["type"]])
        if c["op"] == "rope":
            return B.rope(s["x"], s["table"], positions=s["positions"], first=s["first"], half=c["half"], backward=c["backward"])
        if c["op"] == "append":
            new = B.append_pages(s["k"], s["v"], s["pool"][0], s["pool"][1], s["table"], s["kv_len"], n_new=s["new"], k_rope=s["rotary"],
                                 half=c["half"])
            return s["pool"][0], s["pool"][1], new
        return B.attn_pages(s["q"], s["pool"][0], s["pool"][1], s["table"], s["kv_len"], n_new=s["new"], causal=c["causal"],
                            window=c["window"] or None, sink=c["sink"], want_lse=c["lse"])
    return {"table": _plain_table, "rope": _plain_rope, "append": _plain_append, "attend": _plain_attend}[c["op"]](s)


# --------------------------------------------------------------------------------------- work
def work(case):
    c = case
    if c["op"] == "table":
        n = c["tokens"] * c["pairs"]
        return dict(bytes=n * (4 if c["type"] == "f16" else 8) + (4 * c["tokens"] * c["axes"] if c["axes"] > 1 else 0), flops=3 * n)
    size = 4 if c["type"] == "f32" else 2
    turn = c.get("pairs", 0) * (4 if c.get("table") == "f16" else 8)        # a table's row
    if c["op"] == "rope":
        n = c["seqs"] * c["nodes"]
        return dict(bytes=n * (c["heads"] * 2 * c["dim"] * size + turn), flops=6 * n * c["heads"] * c["pairs"])
    kv, new = _sizes(c)
    if c["op"] == "append":
        return dict(bytes=sum(new) * (c["heads"] * 4 * c["dim"] * size + turn), flops=6 * sum(new) * c["heads"] * c["pairs"])
    nbytes = flops = 0
    for a, b in zip(kv, new):
        seen = pairs = 0
        for i in range(b):
            place = a - b + i
            hi = place + 1 if c["causal"] else a
            lo = max(0, place - c["window"] + 1) if c["window"] else 0
            pairs += hi - lo + min(c["sink"], lo)
        lo = max(0, a - b - c["window"] + 1) if c["window"] else 0
        seen = a - lo + min(c["sink"], lo)
        nbytes += c["heads"] * (2 * seen * c["dim"] * size + 2 * c["group"] * b * c["dim"] * size)
        flops += 4 * c["dim"] * c["heads"] * c["group"] * pairs
    return dict(bytes=nbytes, flops=flops)


# -------------------------------------------------------------------------------------- exact
def _exact_turn(x, cs, half):
    """Rows [.., d] by (cos, sin) as complex numbers, in 64 bits."""
    p, z = cs.shape[-2], torch.view_as_complex(cs.double().contiguous())
    x = x.double().clone()
    if half:
        w = torch.complex(x[..., :p].contiguous(), x[..., p:2 * p].contiguous()) * z
        x[..., :p], x[..., p:2 * p] = w.real, w.imag
    else:
        w = torch.view_as_complex(x[..., :2 * p].reshape(*x.shape[:-1], p, 2).contiguous()) * z
        x[..., :2 * p] = torch.view_as_real(w).flatten(-2)
    return x


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "table":
        pos = s["positions"] if s["positions"] is not None else (torch.arange(c["tokens"], device=DEV) + s["first"])[:, None]
        axis = s["axis"] or [0] * c["pairs"]
        out = torch.empty((c["tokens"], c["pairs"], 2), dtype=torch.float64, device=DEV)
        for p in range(c["pairs"]):
            ang = pos[:, axis[p]].double() * s["freq"][p]
            out[:, p, 0], out[:, p, 1] = ang.cos(), ang.sin()
        return out
    if c["op"] == "rope":
        cs = s["table"].double()
        if c["backward"]:
            cs = cs * torch.tensor([1.0, -1.0], dtype=torch.float64, device=DEV)
        out = torch.empty(s["x"].shape, dtype=torch.float64, device=DEV)
        for b in range(c["seqs"]):
            at = s["positions"][b].long() if c["given"] else torch.arange(c["nodes"], device=DEV) + int(s["first"][b])
            for h in range(c["heads"]):
                out[b, h] = _exact_turn(s["x"][b, h], cs[at], c["half"])
        return out
    kv, new = _sizes(c)
    L = c["page"]
    pages = s["table"].tolist()
    if c["op"] == "append":
        pool = s["pool"].double()
        for b in range(c["seqs"]):
            for a in range(kv[b] // L, -(-(kv[b] + new[b]) // L)):
                # the page's tokens lo..hi-1 of the sequence
                lo, hi = max(a * L, kv[b]), min((a + 1) * L, kv[b] + new[b])
                at = slice(lo - kv[b], hi - kv[b])
                k = s["k"][b, :, at].double()
                if s["rotary"] is not None:
                    k = _exact_turn(k, s["rotary"][lo:hi], c["half"])
                pool[0, :, pages[b][a], lo - a * L:hi - a * L] = k
                pool[1, :, pages[b][a], lo - a * L:hi - a * L] = s["v"][b, :, at].double()
        return pool[0], pool[1], None
    n, H, G, m, d = c["seqs"], c["heads"], c["group"], c["nodes"], c["dim"]
    if n * H * G * m > 20000:
        return None
    out = torch.zeros((n, H * G, m, d), dtype=torch.float64, device=DEV)
    lse = torch.full((n, H * G, m), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(n):
        t = torch.arange(kv[b], device=DEV)
        for h in range(H):
            K, V = (torch.cat([side[h, pages[b][a]] for a in range(-(-kv[b] // L))])[:kv[b]].double() for side in s["pool"])
            for i in range(new[b]):
                place = kv[b] - new[b] + i
                hide = t > place if c["causal"] else t < 0
                if c["window"]:
                    hide = hide | ((t <= place - c["window"]) & (t >= c["sink"]))
                x = (K @ s["q"][b, h * G:(h + 1) * G, i].double().t()).t() / math.sqrt(d)
                x = x.masked_fill(hide, -math.inf)
                z = torch.logsumexp(x, 1)
                out[b, h * G:(h + 1) * G, i] = torch.exp(x - z[:, None]) @ V
                lse[b, h * G:(h + 1) * G, i] = z
    return (out, lse) if c["lse"] else out
