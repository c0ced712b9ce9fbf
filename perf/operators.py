"""Operators over a paged compressed cache whose speed is measured, with their plain forms.

Several sequences keep their compressed tokens in pages of one pool (a page is a chunk of the codec:
page_len tokens with a centroid table of their own), the newest tokens in a bf16 tail, and in every
step a few new tokens (one, or a tree of drafted ones) attend to all of it:

  attend  tree attention of the new tokens over pages, tail and the new tokens themselves
  mask    the trees' parents -> bits of each node's ancestors, and the nodes' depths
  keep    the accepted nodes' K and V appended to the tail
  copy    pages copied (a pool is compacted, a sequence's pages are gathered)

A plain form is the operator's definition in elementary operations.  Sizes are those of
paper_2602_02958_amd/configs.py (heads, chunks as pages, cached tokens), or generic.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128                        # head dimension
DEV = "cuda"


def _attend(name, **kw):
    """`seqs` sequences, `heads` KV heads with `group` query heads each, `nodes` new tokens, up to `tokens` compressed
    tokens in pages of `page`, up to `tail` bf16 tokens.  ragged: lengths differ, down to one token; trees of fewer
    nodes.  tree: a tree of drafted tokens, else each new token sees those before it."""
    c = dict(op="attend", seqs=1, heads=12, group=1, nodes=1, tokens=4096, page=4096, tail=64, K=256, B=64, T=1, S=1,
             bits=2, fp8=False, rope=False, lse=False, tree=False, ragged=False)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def _other(name, op, **kw):
    c = dict(op=op)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one new token of one head over one page: launches and latency
        _attend("token_one_head", heads=1, tokens=4096, page=4096, K=16, T=2, tail=64),
        # a serving batch, one token each, four query heads to a KV head, small pages, the one-round preset
        _attend("token_batch", seqs=16, heads=8, group=4, tokens=32768, page=512, K=64, fp8=True, tail=500, ragged=True),
        # a tree of 64 drafted tokens over a layer of 27 chunks
        _attend("tree_layer", nodes=64, tokens=126360, page=4680, K=256, T=2, tail=1560, tree=True, lse=True),
        # small trees of a batch, shared KV heads, 4-bit levels, an odd tree size, pages that end inside a tile
        _attend("tree_batch_int4", seqs=5, heads=8, group=4, nodes=31, tokens=20000, page=1000, K=256, bits=4, fp8=True,
                tail=777, tree=True, ragged=True),
        # four smoothing stages and the rotary embedding of the cached keys
        _attend("tree_pro_rope", seqs=2, heads=12, nodes=16, tokens=31997, page=4680, K=256, B=16, S=4, fp8=True, tail=300,
                rope=True, tree=True),
        # one token over one layer of the longest rollout
        _attend("token_long_layer", tokens=748800, page=4680, K=256, T=4, tail=4680, lse=True),
        # one tree, once a step for all layers
        _other("mask_one", "mask", seqs=1, nodes=63),
        # many large trees
        _other("mask_batch", "mask", seqs=64, nodes=1000),
        # a step's accepted path of one sequence
        _other("keep_one", "keep", seqs=1, heads=12, nodes=64, tail=1560),
        # accepted paths of a batch over many heads
        _other("keep_batch", "keep", seqs=64, heads=40, nodes=48, tail=512),
        # a few small pages
        _other("copy_small", "copy", units=16, pages=5, page=256, K=16, B=64, T=1, S=1, bits=2, fp8=True),
        # a sequence's chunks of a layer
        _other("copy_chunks", "copy", units=24, pages=20, page=4680, K=256, B=64, T=4, S=1, bits=2, fp8=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


FORMATS = [                    # (K choices, B, T, S, bits, fp8)
    ((16, 64, 256), 64, 2, 1, 2, False), ((64, 100, 256), 32, 3, 1, 2, False), ((128, 256), 64, 4, 1, 2, False),
    ((64, 256), 64, 1, 1, 2, True), ((256,), 16, 1, 4, 2, True), ((256,), 64, 1, 1, 4, True),
    ((512,), 64, 1, 1, 2, True),
]


def draw(rng):
    Ks, Bg, T, S, bits, fp8 = rng.choice(FORMATS)
    fmt = dict(K=rng.choice(Ks), B=Bg, T=T, S=S, bits=bits, fp8=fp8)
    op = rng.choice(["attend"] * 5 + ["mask", "keep", "copy"])
    if op == "mask":
        return _other(None, op, seqs=_log_int(rng, 1, 64), nodes=_log_int(rng, 2, 1000))
    if op == "keep":
        return _other(None, op, seqs=_log_int(rng, 1, 64), heads=_log_int(rng, 1, 40), nodes=_log_int(rng, 1, 64),
                      tail=_log_int(rng, 16, 1560))
    page = 8 * _log_int(rng, 16, 4680 // 8)
    if op == "copy":
        units = 2 * _log_int(rng, 1, 40)
        return _other(None, op, units=units, pages=_log_int(rng, 1, max(1, 2_000_000 // (units * page))), page=page, **fmt)
    heads = _log_int(rng, 1, 40)
    group = rng.choice([1, 1, 2, 4, 8])
    seqs = _log_int(rng, 1, 32)
    nodes = rng.choice([1, 1, _log_int(rng, 2, 128)])
    most = max(page, min(748800, 8_000_000 // (heads * seqs)))          # tokens of all heads: as the longest layer
    most = max(1, min(most, 300_000_000 // (heads * group * seqs * nodes)))
    tokens = _log_int(rng, min(64, most), most)
    return _attend(None, seqs=seqs, heads=heads, group=group, nodes=nodes, tokens=tokens, page=page,
                   tail=_log_int(rng, 1, 1560), rope=rng.random() < 0.25, tree=rng.random() < 0.6,
                   ragged=seqs > 1 and rng.random() < 0.7, **fmt)


# ------------------------------------------------------------------------------------- inputs
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((seed * 1009 + what) % (1 << 62))


def _levels(bits):
    """The code bytes an encoder writes: fields of 2 bits in {0, 1, -1}, or nibbles in -7..7."""
    fields = (0, 1, 3) if bits == 2 else tuple(v & 15 for v in range(-7, 8))
    per = 8 // bits
    idx = torch.cartesian_prod(*[torch.tensor(fields, dtype=torch.int64)] * per)
    return sum(idx[:, i] << (bits * i) for i in range(per)).to(torch.uint8).to(DEV)


def _pool(c, units, n_pages, seed):
    """A pool of encoded pages: centroids [U, P, (S,) K, 128] bf16, ids [U, P*L(, S)], codes [U, P*L, T, 128*bits/8],
    scales [U, P*L, T, 128/B] binary16 or E4M3 bytes.  Later rounds have smaller scales, as in an encoded cache."""
    g = _gen(seed, 1)
    K, S, T, n, G = c["K"], c["S"], c["T"], n_pages * c["page"], D // c["B"]
    cent = torch.randn((units, n_pages, S, K, D), generator=g, device=DEV)
    cent = (cent * 0.4 ** torch.arange(S, device=DEV)[:, None, None]).to(torch.bfloat16)
    ids = torch.randint(0, K, (units, n, S), generator=g, device=DEV, dtype=torch.int16)
    ids = ids.to(torch.uint8) if K <= 256 else ids
    lv = _levels(c["bits"])
    codes = lv[torch.randint(0, lv.numel(), (units, n, T, D * c["bits"] // 8), generator=g, device=DEV, dtype=torch.int16).long()] \
        if units * n * T < 2_000_000 else _codes(lv, units, n, T, D * c["bits"] // 8, g)
    qmax = 1 if c["bits"] == 2 else 7
    if c["fp8"]:
        # 2^-4 .. 2^-1 (seven times less with 4-bit levels)
        lo = 24 if c["bits"] == 2 else 4
        scales = torch.randint(lo, lo + 24, (units, n, T, G), generator=g, device=DEV, dtype=torch.uint8)
    else:
        scales = torch.rand((units, n, T, G), generator=g, device=DEV) * 0.3 + 0.1
        scales = (scales * (1.0 / qmax) * 0.4 ** torch.arange(T, device=DEV)[:, None]).to(torch.float16)
    if S == 1:
        cent, ids = cent[:, :, 0].contiguous(), ids[:, :, 0].contiguous()
    return dict(cent=cent, ids=ids, codes=codes, scales=scales)


def _codes(lv, units, n, T, width, g):
    out = torch.empty((units, n, T, width), dtype=torch.uint8, device=DEV)
    for u in range(units):
        out[u] = lv[torch.randint(0, lv.numel(), (n, T, width), generator=g, device=DEV, dtype=torch.int16).int()]
    return out


def _rope_table(n):
    freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) / (D // 2))
    ang = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * freq[None]
    return torch.stack([ang.cos(), ang.sin()], -1).to(torch.float16).contiguous()


def _lengths(c, most, what, low):
    """Lengths of the sequences, known from the case alone: all `most`, or spread over low..most with both ends among them."""
    n = c["seqs"]
    if not c.get("ragged") or n == 1:
        return [most] * n
    out = [low + ((i * 7919 + what * 104729 + 31 * most) % 1000) * (most - low) // 1000 for i in range(n)]
    out[0], out[n - 1] = most, low
    return out


def _sizes(c):
    return _lengths(c, c["tokens"], 1, 1), _lengths(c, c["tail"], 2, 0), _lengths(c, c["nodes"], 3, 1)


def _parents(seqs, nodes, sizes, seed):
    """A draft tree per sequence, parents before children, most of them recent; -2 behind the tree's last node."""
    g = _gen(seed, 2)
    i = torch.arange(nodes, device=DEV)
    back = 1 + (torch.rand((seqs, nodes), generator=g, device=DEV) ** 2 * 7).long()
    p = torch.clamp(i - back, min=-1).to(torch.int32)
    return torch.where(i[None] < torch.tensor(sizes, device=DEV)[:, None], p, -2).to(torch.int32).contiguous()


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c, g = case, _gen(seed, 3)
    if c["op"] == "mask":
        sizes = [max(1, c["nodes"] - i % 5) for i in range(c["seqs"])]
        return dict(case=c, parents=_parents(c["seqs"], c["nodes"], sizes, seed))
    if c["op"] == "keep":
        # the model's K and V of the new tokens, [sequence, token, head, 128]; paths of half a tree or less
        n, h, m = c["seqs"], c["heads"], c["nodes"]
        k, v = (torch.randn((n, m, h, D), generator=g, device=DEV).to(torch.bfloat16).transpose(1, 2) for _ in range(2))
        tail = torch.randn((n, 2 * h, c["tail"] + m, D), generator=g, device=DEV).to(torch.bfloat16)
        order = torch.rand((n, m), generator=g, device=DEV).argsort(1)[:, :(m + 1) // 2].sort(1)[0]
        keep = torch.randint(1, (m + 1) // 2 + 1, (n,), generator=g, device=DEV)
        length = torch.randint(0, c["tail"] + 1, (n,), generator=g, device=DEV)
        return dict(case=c, k=k, v=v, tail_k=tail[:, :h], tail_v=tail[:, h:], tail=tail, path=order.to(torch.int32).contiguous(),
                    keep=keep.to(torch.int32), length=length.to(torch.int32))
    if c["op"] == "copy":
        # the pages go behind each other at the pool's end
        n = c["pages"]
        pool = _pool(c, c["units"], 2 * n + 1, seed)
        src = torch.randperm(n + 1, generator=g, device=DEV)[:n].tolist()
        return dict(case=c, pool=pool, src=src, dst=list(range(n + 1, 2 * n + 1)))
    n, h, m, L = c["seqs"], c["heads"], c["nodes"], c["page"]
    kv, tails, nodes = _sizes(c)
    per = -(-c["tokens"] // L)
    used = [-(-x // L) for x in kv]
    pool = _pool(c, 2 * h, sum(used) + 1, seed)
    # a sequence's pages lie anywhere in the pool; behind its last page a table holds page 0
    free = torch.randperm(sum(used) + 1, generator=g, device=DEV).tolist()
    table = [[free.pop() for _ in range(u)] + [0] * (per - u) for u in used]
    q = torch.randn((n, m, h * c["group"], D), generator=g, device=DEV).to(torch.bfloat16).transpose(1, 2)
    k, v = (torch.randn((n, m, h, D), generator=g, device=DEV).to(torch.bfloat16).transpose(1, 2) for _ in range(2))
    tail = torch.randn((n, 2 * h, c["tail"] + m, D), generator=g, device=DEV).to(torch.bfloat16)
    st = dict(case=c, q=q, table=_int32(table), kv_len=_int32(kv), tail_k=tail[:, :h], tail_v=tail[:, h:], tail_len=_int32(tails),
              k=k, v=v, nodes=_int32(nodes), rope=_rope_table(per * L) if c["rope"] else None, mask=None,
              kside={x: t[:h] for x, t in pool.items()}, vside={x: t[h:] for x, t in pool.items()})
    if c["tree"]:
        par = _parents(n, m, nodes, seed)
        st["mask"] = _plain_mask(par)[0]
    return st


# ------------------------------------------------------------------------------- plain forms
def _plain_mask(parents):
    """Ancestors by squaring the parent relation: reach = (1 + A)^(2^k), ten squarings for up to 1024 nodes."""
    n, m = parents.shape
    i = torch.arange(m, device=parents.device)
    hole = (parents < -1) | (parents >= i)
    up = ((parents.long()[:, :, None] == i) & ~hole[:, :, None]).float()
    reach = up + torch.eye(m, device=parents.device)
    for _ in range(max(1, (m - 1).bit_length())):
        reach = ((reach @ reach) > 0).float()
    bad = (reach * hole[:, None, :].float()).amax(2) > 0                    # a hole, or a node below one
    reach = reach * (~bad)[:, :, None].float()
    depth = torch.where(bad, -1, reach.sum(2).int() - 1).to(torch.int32)
    words = -(-m // 32)
    bits = torch.zeros((n, m, words * 32), dtype=torch.int64, device=parents.device)
    bits[:, :, :m] = reach.long()
    w = (bits.view(n, m, words, 32) << torch.arange(32, device=parents.device)).sum(3)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32), depth


def _scale_values(s):
    """Scales as numbers: binary16, or the OCP E4M3 layout."""
    if s.dtype != torch.uint8:
        return s.float()
    b = s.int()
    e, m = (b >> 3) & 15, (b & 7).float()
    return torch.where(e > 0, (1 + m / 8) * torch.exp2(e.float() - 7), m / 8 * 2.0 ** -6)


def _plain_side(c, side, table):
    """fp32 values of the sequences' pages, [H, seqs, pages * L, 128]."""
    H, L, T, S = c["heads"], c["page"], c["T"], c["S"]
    n, per = table.shape
    at = table.long().reshape(-1)
    P = side["ids"].shape[1] // L
    pick = lambda t: t.reshape(H, P, L, *t.shape[2:])[:, at]                # noqa: E731
    ids = pick(side["ids"]).long().reshape(H, n * per, L, S)
    cent = side["cent"].reshape(H, P, S, c["K"], D)[:, at].float()
    codes, scales = pick(side["codes"]), _scale_values(pick(side["scales"]))
    x = sum(torch.gather(cent[:, :, s], 2, ids[..., s, None].expand(-1, -1, -1, D)) for s in range(S))
    b = c["bits"]
    shift = torch.arange(0, 8, b, device=DEV, dtype=torch.uint8)
    for t in range(T):
        f = ((codes[:, :, :, t, :, None] >> shift) & ((1 << b) - 1)).reshape(H, n * per, L, D).to(torch.int8)
        f = torch.where(f >= 1 << (b - 1), f - (1 << b), f)
        x = x + f.float() * scales[:, :, :, t].repeat_interleave(c["B"], -1)
    return x.reshape(H, n, per * L, D)


def _plain_attend(s):
    c = s["case"]
    H, G, m = c["heads"], c["group"], c["nodes"]
    K, V = (_plain_side(c, s[x], s["table"]).transpose(0, 1) for x in ("kside", "vside"))        # [n, H, tokens, 128]
    if s["rope"] is not None:
        cos, sin = s["rope"].float().unbind(-1)
        a, b = K[..., 0::2], K[..., 1::2]
        K = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    K = torch.cat([K, s["tail_k"].float(), s["k"].float()], 2)
    V = torch.cat([V, s["tail_v"].float(), s["v"].float()], 2)
    n = K.shape[0]
    i = torch.arange(m, device=DEV)
    seen = (i[None, :] <= i[:, None]).expand(n, -1, -1) if s["mask"] is None else \
        ((s["mask"][..., None] >> torch.arange(32, device=DEV)) & 1).flatten(-2)[..., :m].bool()
    ahead = lambda t, w: (torch.arange(w, device=DEV) < t[:, None])[:, None].expand(-1, m, -1)   # noqa: E731
    row = i[None] < s["nodes"][:, None]
    see = torch.cat([ahead(s["kv_len"], s["table"].shape[1] * c["page"]), ahead(s["tail_len"], s["tail_k"].shape[2]),
                     seen & row[:, None, :]], 2) & row[:, :, None]
    x = torch.matmul(s["q"].float().reshape(n, H, G * m, D), K.transpose(2, 3)) * (1.0 / math.sqrt(D))
    x = torch.where(see[:, None, None], x.reshape(n, H, G, m, -1), -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(n, H, G * m, -1), V).reshape(n, H, G, m, D) / total.clamp(min=1e-38)
    o = torch.where(row[:, None, None, :, None], o, 0.0).reshape(n, H * G, m, D).to(torch.bfloat16)
    if not c["lse"]:
        return o
    return o, (top + torch.log(total)).reshape(n, H * G, m)


def _plain_keep(s):
    """Rows of the tail picked from the new tokens where a kept one goes, else left; the tail as a new state."""
    m = s["path"].shape[1]
    i = torch.arange(m, device=DEV)
    n, U, R, _ = s["tail"].shape
    src = torch.cat([s["k"], s["v"]], 1)
    rows = torch.gather(src, 2, s["path"].long()[:, None, :, None].expand(-1, U, -1, D))
    at = s["length"].long()[:, None] + i
    live = i[None] < s["keep"][:, None]
    pos = torch.arange(R, device=DEV)
    hit = (pos[None, :, None] == at[:, None, :]) & live[:, None, :]           # [n, R, m]
    which = hit.int().argmax(2)
    new = torch.gather(rows, 2, which[:, None, :, None].expand(-1, U, -1, D))
    s["tail"].copy_(torch.where(hit.any(2)[:, None, :, None], new, s["tail"]))
    return s["tail"], s["length"] + s["keep"]


def _dst_pages(s):
    """The copied pages, whole (they are the pool's last)."""
    c, p = s["case"], s["pool"]
    a = s["dst"][0]
    return [p["cent"][:, a:]] + [p[x][:, a * c["page"]:] for x in ("ids", "codes", "scales")]


def _plain_copy(s):
    c, p = s["case"], s["pool"]
    src, dst = (torch.tensor(x, device=DEV) for x in (s["src"], s["dst"]))
    p["cent"][:, dst] = p["cent"][:, src]
    for x in ("ids", "codes", "scales"):
        t = p[x].view(c["units"], -1, c["page"], *p[x].shape[2:])
        t[:, dst] = t[:, src]
    return _dst_pages(s)


# ---------------------------------------------------------------------------------------- run
def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2602_02958_amd import binding as B
        enc = lambda p: B.Encoded(p["cent"], p["ids"], p["codes"], p["scales"], c["page"], c["S"])     # noqa: E731
        if c["op"] == "mask":
            return B.tree_mask(s["parents"])
        if c["op"] == "keep":
            new = B.keep_nodes(s["k"], s["v"], s["path"], s["keep"], s["tail_k"], s["tail_v"], s["length"])
            return s["tail"], new
        if c["op"] == "copy":
            B.copy_pages(enc(s["pool"]), s["src"], s["dst"])
            return _dst_pages(s)
        return B.attn_tree(s["q"], enc(s["kside"]), enc(s["vside"]), s["table"], s["kv_len"], s["k"], s["v"],
                           tail_k=s["tail_k"], tail_v=s["tail_v"], tail_len=s["tail_len"], n_nodes=s["nodes"],
                           mask=s["mask"], k_rope=s["rope"], want_lse=c["lse"])
    if c["op"] == "mask":
        return _plain_mask(s["parents"])
    if c["op"] == "keep":
        return _plain_keep(s)
    if c["op"] == "copy":
        return _plain_copy(s)
    return _plain_attend(s)


# --------------------------------------------------------------------------------------- work
def _page_bytes(c):
    """Bytes of a token and of a page's tables."""
    per = c["S"] * (2 if c["K"] > 256 else 1) + c["T"] * (D * c["bits"] // 8 + D // c["B"] * (1 if c["fp8"] else 2))
    return per, c["S"] * c["K"] * D * 2


def work(case):
    c = case
    if c["op"] == "mask":
        n, m = c["seqs"], c["nodes"]
        return dict(bytes=4 * n * m * (2 + -(-m // 32)), flops=n * m * -(-m // 32))
    if c["op"] == "keep":
        # about a quarter of the nodes are kept: read and written
        return dict(bytes=c["seqs"] * 2 * c["heads"] * max(1, (c["nodes"] + 1) // 4) * D * 2 * 2, flops=0)
    token, table = _page_bytes(c)
    if c["op"] == "copy":
        return dict(bytes=2 * c["units"] * c["pages"] * (c["page"] * token + table), flops=0)
    nbytes = flops = 0
    H, G = c["heads"], c["group"]
    for kv, tail, m in zip(*_sizes(c)):
        nbytes += 2 * H * (kv * token + -(-kv // c["page"]) * table + (tail + m) * D * 2) + 2 * H * G * m * D * 2
        nbytes += kv * D * 2 if c["rope"] else 0
        flops += 4 * D * H * G * m * (kv + tail + (m + 1) // 2)
    return dict(bytes=nbytes, flops=flops)


# -------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The attention in 64 bits, one sequence and head at a time; the other operators give whole numbers or bytes."""
    c = case
    if c["op"] != "attend":
        return None
    s = prepare(case, seed)
    kv, tails, nodes = _sizes(c)
    n, H, G, m, L, S, T, b = c["seqs"], c["heads"], c["group"], c["nodes"], c["page"], c["S"], c["T"], c["bits"]
    out = torch.zeros((n, H * G, m, D), dtype=torch.float64, device=DEV)
    lse = torch.full((n, H * G, m), -math.inf, dtype=torch.float64, device=DEV)
    e4m3 = torch.tensor([(1 + (v & 7) / 8) * 2.0 ** ((v >> 3) - 7) if v >= 8 else (v & 7) * 2.0 ** -9 for v in range(128)],
                        dtype=torch.float64, device=DEV)
    per = 8 // b
    value = [v - (1 << b) if v >= 1 << (b - 1) else v for v in range(1 << b)]
    lut = torch.tensor([[value[(v >> (b * i)) & ((1 << b) - 1)] for i in range(per)] for v in range(256)],
                       dtype=torch.float64, device=DEV)

    def page(side, h, p, count):
        """The first `count` tokens of page p."""
        rows = slice(p * L, p * L + count)
        ids = side["ids"][h, rows].reshape(count, S).long()
        table = side["cent"][h, p].reshape(S, c["K"], D).double()
        x = torch.zeros((count, D), dtype=torch.float64, device=DEV)
        for st in range(S):
            x += table[st].index_select(0, ids[:, st])
        lev = lut.index_select(0, side["codes"][h, rows].reshape(-1).int()).reshape(count, T, D // c["B"], c["B"])
        sc = side["scales"][h, rows]
        sc = e4m3[sc.long()] if c["fp8"] else sc.double()
        return x + (lev * sc[..., None]).sum(1).reshape(count, D)

    for j in range(n):
        pages = s["table"][j].tolist()
        # what node i sees of the nodes, bit by bit
        if s["mask"] is None:
            vis = torch.ones((m, m), dtype=torch.bool).tril()
        else:
            words = s["mask"][j].cpu().tolist()
            vis = torch.tensor([[(words[i][k // 32] >> (k % 32)) & 1 for k in range(m)] for i in range(m)], dtype=torch.bool)
        vis = vis[:nodes[j], :nodes[j]].to(DEV)
        for h in range(H):
            def keys(side):
                parts = [page(s[side], h, pages[a // L], min(L, kv[j] - a)) for a in range(0, kv[j], L)]
                return torch.cat(parts) if parts else torch.zeros((0, D), dtype=torch.float64, device=DEV)
            K, V = keys("kside"), keys("vside")
            if s["rope"] is not None:
                z = torch.view_as_complex(s["rope"][:kv[j]].double().contiguous())
                K = torch.view_as_real(torch.view_as_complex(K.view(kv[j], D // 2, 2)) * z).reshape(kv[j], D)
            K = torch.cat([K, s["tail_k"][j, h, :tails[j]].double(), s["k"][j, h, :nodes[j]].double()])
            V = torch.cat([V, s["tail_v"][j, h, :tails[j]].double(), s["v"][j, h, :nodes[j]].double()])
            old = kv[j] + tails[j]
            for u in range(G):
                x = s["q"][j, h * G + u, :nodes[j]].double() @ K.t() / math.sqrt(D)
                x[:, old:].masked_fill_(~vis, -math.inf)
                z = torch.logsumexp(x, 1)
                out[j, h * G + u, :nodes[j]] = torch.exp(x - z[:, None]) @ V
                lse[j, h * G + u, :nodes[j]] = z
    return (out, lse) if c["lse"] else out
