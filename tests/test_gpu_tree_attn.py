"""attn_tree on the GPU against the attention in 64 bits (tree_util.reference, which derives the tolerances)."""
import math

import pytest
import torch

from tree_util import D, Pool, bits_of, plain_mask, random_parents, reference

pytestmark = pytest.mark.gpu
B = pytest.importorskip("paper_2602_02958_amd.binding")


def make(pool, H, g, m, kv, tails, nodes, seed=0, tree=True, R=None, rope=False):
    """Inputs of a step on the host: lists of lengths, one entry per sequence."""
    gen = torch.Generator().manual_seed(seed + 100)
    n = len(kv)
    R = max(tails) + 3 if R is None else R
    q = torch.randn(n, m, H * g, D, generator=gen).to(torch.bfloat16).transpose(1, 2)
    k, v = (torch.randn(n, m, H, D, generator=gen).to(torch.bfloat16).transpose(1, 2) for _ in range(2))
    tail = torch.randn(n, 2 * H, R, D, generator=gen).to(torch.bfloat16)
    per = max(1, max(-(-x // pool.L) for x in kv))
    table = torch.stack([torch.randperm(pool.pages, generator=gen)[:per] if per <= pool.pages else
                         torch.randint(0, pool.pages, (per,), generator=gen) for _ in range(n)]).to(torch.int32)
    see = plain_mask(random_parents(n, m, seed))[0] if tree else torch.ones(m, m).tril().bool().expand(n, m, m)
    if rope:
        ang = torch.rand(per * pool.L, D // 2, generator=gen, dtype=torch.float64) * 6.3
        rope = torch.stack([ang.cos(), ang.sin()], -1).to(torch.float16)
    else:
        rope = None
    return dict(q=q, k_new=k, v_new=v, tail=tail, table=table, kv=kv, tails=tails, nodes=nodes, see=see, tree=tree, rope=rope, H=H)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def call(pool, x, scratch=None, **kw):
    H, c = x["H"], "cuda"
    tail = x["tail"].to(c)
    # (strided views keep their strides on the way to the device)
    q, k, v = (x[t].transpose(1, 2).contiguous().to(c).transpose(1, 2) for t in ("q", "k_new", "v_new"))
    return B.attn_tree(q, pool.encoded(0, H), pool.encoded(H, 2 * H), x["table"].to(c), ints(x["kv"]), k, v, tail_k=tail[:, :H],
                       tail_v=tail[:, H:], tail_len=ints(x["tails"]), n_nodes=ints(x["nodes"]), want_lse=True,
                       mask=bits_of(x["see"]).to(c) if x["tree"] else None, k_rope=None if x["rope"] is None else x["rope"].to(c),
                       scratch=scratch, **kw)


def check(pool, x, got, scale=None):
    H = x["H"]
    out, lse, tol, ltol = reference(x["q"], pool, H, x["table"], x["kv"], x["k_new"], x["v_new"], x["tail"][:, :H], x["tail"][:, H:],
                                    x["tails"], x["nodes"], x["see"], x["rope"], scale)
    o, z = got[0].double().cpu(), got[1].double().cpu()
    empty = torch.isneginf(lse)
    assert torch.equal(torch.isneginf(z), empty)
    assert (o[empty] == 0).all()
    err = (o - out).abs()
    assert torch.isfinite(o).all() and (err <= tol + 1e-30).all(), f"out off by {(err / (tol + 1e-30)).max():.3g} of its bound"
    lerr = torch.where(empty, torch.zeros_like(lse), (z - lse).abs())
    assert (lerr <= ltol + 1e-30).all(), f"lse off by {(lerr / (ltol + 1e-30)).max():.3g} of its bound"
    # the bounds above are for the worst case; together the errors are far below it: half a step of bf16 and as much again
    assert (o - out).norm() <= 2.0 ** -7 * out.norm()


NO_SCRATCH = torch.empty(0, dtype=torch.uint8)

FORMATS = [dict(T=1), dict(T=2, K=64), dict(T=3, B=32, K=100), dict(T=4, K=256), dict(T=1, fp8=True, K=256), dict(T=1, B=16, S=4, fp8=True),
           dict(T=1, bits=4, fp8=True), dict(T=1, K=512, fp8=True), dict(T=8, B=128), dict(T=2, bits=4), dict(T=3, S=2, K=300, B=16),
           dict(T=5, fp8=True, B=16), dict(T=2, S=3, bits=4, B=32), dict(K=1, T=1)]


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: "-".join(f"{k}{v}" for k, v in f.items()))
@pytest.mark.parametrize("divided", [True, False])
@pytest.mark.parametrize("rope", [False, True])
def test_formats(fmt, divided, rope):
    pool = Pool(4, 5, 72, seed=1, **fmt)
    x = make(pool, 2, 2, 7, [300, 72, 5], [33, 0, 9], [7, 3, 7], seed=2, rope=rope)
    check(pool, x, call(pool, x, scratch=None if divided else NO_SCRATCH.cuda()))


LENGTHS = [   # page_len, kv, tail, nodes
    (32, [1], [0], [1]), (32, [32], [0], [1]), (32, [33, 31, 64], [1, 32, 33], [1, 1, 1]),
    (8, [8, 9, 7, 0], [0, 0, 0, 0], [1, 2, 3, 4]), (1, [5, 3], [0, 2], [2, 2]), (100, [1000, 1, 0], [0, 70, 0], [5, 5, 5]),
    (33, [231], [31], [33]), (4680, [4680], [64], [1]), (40, [0, 0, 0], [0, 5, 0], [3, 0, 1]), (512, [3000, 17], [511, 0], [2, 1]),
]


@pytest.mark.parametrize("page,kv,tails,nodes", LENGTHS, ids=str)
@pytest.mark.parametrize("tree", [True, False])
def test_lengths(page, kv, tails, nodes, tree):
    pool = Pool(2, max(2, max(-(-x // page) for x in kv)), page, T=2, K=32, B=32, seed=3)
    x = make(pool, 1, 1, max(nodes), kv, tails, nodes, seed=4, tree=tree)
    check(pool, x, call(pool, x))


@pytest.mark.parametrize("H,g,m", [(1, 1, 1), (3, 1, 16), (1, 4, 5), (2, 3, 11), (1, 8, 8), (2, 1, 63), (1, 5, 33), (1, 2, 100), (1, 1, 257)])
@pytest.mark.parametrize("divided", [True, False])
def test_rows(H, g, m, divided):
    """Blocks of 16, 32 and 64 query rows, several of them, and the last one not full."""
    pool = Pool(2 * H, 6, 56, T=1, K=16, fp8=True, seed=5)
    x = make(pool, H, g, m, [330, 100], [20, 45], [m, max(1, m // 2)], seed=6)
    check(pool, x, call(pool, x, scratch=None if divided else NO_SCRATCH.cuda()))


@pytest.mark.parametrize("spread", [1e-4, 1.0, 30.0])
@pytest.mark.parametrize("qs", [1e-30, 1.0, 1e20])
def test_magnitudes(spread, qs):
    """Queries of any magnitude (the scale that keeps the scores in reach goes the other way), small and large stored values."""
    pool = Pool(2, 4, 64, T=2, K=16, seed=7, spread=spread)
    x = make(pool, 1, 2, 3, [250], [10], [3], seed=8)
    for t in ("k_new", "v_new", "tail"):
        x[t] = (x[t].float() * spread).to(torch.bfloat16)
    x["q"] = (x["q"].float() * qs).to(torch.bfloat16)
    scale = 0.1 / qs / spread
    check(pool, x, call(pool, x, softmax_scale=scale), scale=scale)


def test_far_apart_scores():
    """Weights far below the largest, and a maximum that arrives last: the running reference moves at every size of step."""
    pool = Pool(2, 3, 96, T=1, K=8, seed=9)
    for steps in ([1.0, 4.0, 9.0], [9.0, 4.0, 1.0], [0.0, 40.0, 39.0]):
        x = make(pool, 1, 1, 4, [288], [90], [4], seed=10)
        for i, s in enumerate(steps):
            x["tail"][0, 0, 30 * i:30 * i + 30] = (s * x["q"][0, 0, 1].float() / 12).to(torch.bfloat16)
        check(pool, x, call(pool, x))


def test_unseen_places_may_hold_anything():
    """Holes of a tree, rows behind a tree's nodes, the tail behind its length, table entries and page tokens behind a sequence's end."""
    pool = Pool(2, 4, 40, T=2, K=16, seed=11)
    x = make(pool, 1, 2, 37, [90, 40], [7, 0], [37, 20], seed=12, R=50)
    par = random_parents(2, 37, 12)
    par[0, 5] = -2                                         # a hole, and what hangs below it
    par[1, 3] = 9
    see, depth = plain_mask(par, [37, 20])
    x["see"] = see
    clean = call(pool, x)
    holes = depth < 0
    for t in ("k_new", "v_new"):
        for b in range(2):
            x[t][b, :, holes[b]] = float("nan")
    x["tail"][0, :, 7:] = float("inf")
    x["tail"][1] = float("nan")
    x["table"][0, 3:] = 1 << 30
    x["table"][1, 1:] = -5
    dirty = call(pool, x)
    assert torch.equal(clean[0], dirty[0]) and torch.equal(clean[1], dirty[1])
    for t in ("k_new", "v_new", "tail"):
        x[t] = torch.nan_to_num(x[t], 0.0, 0.0, 0.0)
    check(pool, x, dirty)


def test_a_page_number_outside_the_pool_reads_the_nearest_page():
    pool = Pool(2, 3, 32, T=1, seed=13)
    x = make(pool, 1, 1, 2, [90], [0], [2], seed=14)
    x["table"][0] = torch.tensor([-7, 1, 99])
    check(pool, x, call(pool, x))                          # (the reference clamps them, as the interface says)


def test_lengths_outside_their_range_are_clamped():
    pool = Pool(2, 2, 32, T=1, seed=15)
    x = make(pool, 1, 1, 3, [64, 0], [5, 0], [3, 0], seed=16, R=5)
    want = call(pool, x)
    x.update(kv=[1 << 30, -4], tails=[77, -1], nodes=[9, -3])
    got = call(pool, x)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_strides_and_results_in_a_view():
    """A fused projection's q, k and v as views of one tensor, and a result that goes into a view of another layout."""
    pool = Pool(4, 4, 48, T=2, K=16, seed=17)
    H, g, m = 2, 3, 5
    x = make(pool, H, g, m, [150, 97], [12, 30], [5, 4], seed=18)
    want = call(pool, x)
    n = 2
    qkv = torch.full((n, m, H * g + 2 * H + 1, D + 8), float("nan"), dtype=torch.bfloat16)
    for lo, hi, t in ((0, H * g, "q"), (H * g, H * g + H, "k_new"), (H * g + H, H * g + 2 * H, "v_new")):
        qkv[:, :, lo:hi, :D] = x[t].transpose(1, 2)
    qkv = qkv.cuda()
    view = lambda lo, hi: qkv[:, :, lo:hi, :D].transpose(1, 2)
    tail = x["tail"].cuda()
    room = torch.full((n, m, H * g, D + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[..., :D].transpose(1, 2)
    got = B.attn_tree(view(0, H * g), pool.encoded(0, H), pool.encoded(H, 2 * H), x["table"].cuda(), ints(x["kv"]),
                      view(H * g, H * g + H), view(H * g + H, H * g + 2 * H), tail_k=tail[:, :H], tail_v=tail[:, H:],
                      tail_len=ints(x["tails"]), n_nodes=ints(x["nodes"]), mask=bits_of(x["see"]).cuda(), want_lse=True, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert (room[..., D:] == 7.0).all()


def test_without_pages_and_without_a_tail():
    pool = Pool(2, 1, 32, T=1, seed=19)
    x = make(pool, 1, 2, 6, [0], [0], [6], seed=20)
    q, k, v = (x[t].cuda() for t in ("q", "k_new", "v_new"))
    got = B.attn_tree(q, pool.encoded(0, 1), pool.encoded(1, 2), None, None, k, v, mask=bits_of(x["see"]).cuda(), want_lse=True)
    check(pool, x, got)
    # nothing to see at all: no node sees any
    none = torch.zeros(1, 6, 1, dtype=torch.int32, device="cuda")
    o, z = B.attn_tree(q, pool.encoded(0, 1), pool.encoded(1, 2), None, None, k, v, mask=none, want_lse=True)
    assert (o == 0).all() and torch.isneginf(z).all()
    # no sequence, no node
    assert B.attn_tree(q[:0], pool.encoded(0, 1), pool.encoded(1, 2), None, None, k[:0], v[:0]).shape == (0, 2, 6, D)
    assert B.attn_tree(q[:, :, :0], pool.encoded(0, 1), pool.encoded(1, 2), None, None, k[:, :, :0], v[:, :, :0]).shape == (1, 2, 0, D)


def test_equal_calls_give_equal_bits_also_on_other_streams_and_in_a_replayed_graph():
    pool = Pool(4, 6, 200, T=2, K=32, seed=21)
    H = 2
    x = make(pool, H, 1, 8, [1200, 777], [60, 0], [8, 8], seed=22)
    args = [x["q"].cuda(), pool.encoded(0, H), pool.encoded(H, 4), x["table"].cuda(), ints(x["kv"]), x["k_new"].cuda(), x["v_new"].cuda()]
    tail = x["tail"].cuda()
    kw = dict(tail_k=tail[:, :H], tail_v=tail[:, H:], tail_len=ints(x["tails"]), mask=bits_of(x["see"]).cuda(), want_lse=True)
    want = [t.clone() for t in B.attn_tree(*args, **kw)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            outs += [B.attn_tree(*args, **kw) for _ in range(3)]
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0], want[0]) and torch.equal(o[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.attn_tree(*args, **kw)
    kv2 = ints([900, 1])
    for lens in (ints(x["kv"]), kv2, ints(x["kv"])):
        args[4].copy_(lens)
        got[0].fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = B.attn_tree(*args, **kw)
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
    assert torch.equal(got[0], want[0])


def test_offsets_beyond_32_bits():
    """A unit whose codes take more than 4 GiB: the pages lie at its end."""
    L, T, K = 4096, 4, 16
    pages = (1 << 32) // (L * T * 32) + 3
    small = Pool(2, 2, L, T=T, K=K, B=128, seed=23)
    e = B.alloc_cache(2, pages * L, L, K, 128, T)
    src = small.encoded(0, 2)
    B.copy_pages(src, [0, 1], [pages - 1, pages - 2], into=e)
    half = lambda lo: B.Encoded(e.centroids[lo:lo + 1], e.ids[lo:lo + 1], e.codes[lo:lo + 1], e.scales[lo:lo + 1], L)
    x = make(small, 1, 1, 2, [L + 100], [0], [2], seed=24)
    x["table"] = torch.tensor([[0, 1]], dtype=torch.int32)
    table = ints([[pages - 1, pages - 2]])
    got = B.attn_tree(x["q"].cuda(), half(0), half(1), table, ints(x["kv"]), x["k_new"].cuda(), x["v_new"].cuda(),
                      mask=bits_of(x["see"]).cuda(), want_lse=True)
    check(small, x, got)


def test_an_id_beyond_the_table_reads_its_last_row():
    pool = Pool(2, 2, 64, T=1, K=10, seed=25)
    x = make(pool, 1, 1, 1, [100], [0], [1], seed=26)
    pool.ids[0, 5] = 255
    pool.ids[1, 70] = 10
    got = call(pool, x)
    pool.ids[0, 5] = 9
    pool.ids[1, 70] = 9
    check(pool, x, got)
    want = call(pool, x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
