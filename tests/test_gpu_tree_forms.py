"""attn_tree on the GPU: every stored format that has kernels of its own with every number of rows that takes another form, the
ways a call is divided, and tables, addresses and streams that the other tests leave out.  Tolerances: tree_util.reference."""
import pytest
import torch

from tree_util import D, Pool, bits_of, plain_mask, random_parents
from test_gpu_tree_attn import NO_SCRATCH, check, call, ints, make

pytestmark = pytest.mark.gpu
B = pytest.importorskip("paper_2602_02958_amd.binding")

PACKED = [dict(T=1, fp8=True), dict(T=1, B=16, fp8=True), dict(T=1, B=16, S=4, fp8=True), dict(T=1, bits=4, fp8=True),
          dict(T=1, B=16, S=4, bits=4, fp8=True), dict(T=1), dict(T=2), dict(T=2, B=32), dict(T=3), dict(T=3, B=32), dict(T=4),
          dict(T=4, B=32)]
GENERAL = [dict(T=2, fp8=True), dict(T=8, B=128), dict(T=2, S=2, bits=4, B=16)]
name = lambda f: "-".join(f"{k}{v}" for k, v in f.items())


@pytest.mark.parametrize("fmt", PACKED + GENERAL, ids=name)
@pytest.mark.parametrize("g,m", [(1, 16), (4, 5), (8, 4), (5, 8), (8, 8), (13, 5), (4, 32), (3, 43)])
@pytest.mark.parametrize("rope", [False, True])
def test_rows_of_every_format(fmt, g, m, rope):
    """16, 20, 32, 40, 64, 65, 128 and 129 rows; pages that end inside a tile, one that holds a token, a sequence without any."""
    pool = Pool(2, 6, 50, K=20, seed=31, **fmt)
    x = make(pool, 1, g, m, [251, 50, 0], [9, 40, 3], [m, max(1, m - 2), m], seed=32, rope=rope)
    check(pool, x, call(pool, x))


@pytest.mark.parametrize("fmt", [dict(T=1, fp8=True), dict(T=2), dict(T=4, B=32), dict(T=1, B=16, S=4, fp8=True)], ids=name)
@pytest.mark.parametrize("K", [255, 256, 257, 512])
@pytest.mark.parametrize("g,m", [(1, 3), (2, 12), (3, 33)])
def test_tables_of_every_size(fmt, K, g, m):
    pool = Pool(2, 3, 77, K=K, seed=33, **fmt)
    x = make(pool, 1, g, m, [200], [5], [m], seed=34)
    check(pool, x, call(pool, x))


@pytest.mark.parametrize("fmt", [dict(T=1, B=16, S=4, fp8=True), dict(T=1, B=16, S=4, bits=4, fp8=True), dict(T=1, fp8=True),
                                 dict(T=2, S=3, B=32)], ids=name)
@pytest.mark.parametrize("m,rope", [(1, False), (20, False), (70, False), (1, True), (20, True), (40, True)])
def test_long_sequences_in_many_parts(fmt, m, rope):
    """Long enough for more than sixteen parts of one sequence beside a short one and an empty one: parts that walk a range in turns."""
    pool = Pool(2, 7, 900, K=40, seed=35, **fmt)
    x = make(pool, 1, 1, m, [6200, 33, 0], [20, 0, 0], [m, 1, 1], seed=36, rope=rope)
    check(pool, x, call(pool, x))


@pytest.mark.parametrize("n,pages", [(64, 8), (200, 8), (256, 3), (300, 2)])
@pytest.mark.parametrize("divided", [True, False])
def test_many_ragged_sequences(n, pages, divided):
    """More sequences than a wavefront has lanes, some empty, some of one token, some full; 300 are not divided."""
    pool = Pool(2, 9, 100, K=8, T=1, fp8=True, seed=37)
    g = torch.Generator().manual_seed(38)
    kv = torch.randint(0, pages * 100 + 1, (n,), generator=g).tolist()
    tails, nodes = torch.randint(0, 20, (n,), generator=g).tolist(), torch.randint(0, 3, (n,), generator=g).tolist()
    kv[:4], tails[:4], nodes[:4] = [0, 0, pages * 100, 1], [0, 3, 19, 0], [2, 0, 2, 1]
    kv[n - 1], kv[n // 2:n // 2 + 5] = pages * 100, [0] * 5
    x = make(pool, 1, 2, 2, kv, tails, nodes, seed=39)
    check(pool, x, call(pool, x, scratch=None if divided else NO_SCRATCH.cuda()))


def test_scratch_that_is_too_small_or_dirty():
    pool = Pool(4, 6, 200, K=16, T=2, seed=40)
    x = make(pool, 2, 2, 4, [1100, 300], [9, 0], [4, 3], seed=41)
    want = call(pool, x)
    need = B.attn_tree_scratch(pool.encoded(0, 2), 2, 2, 4, x["table"].shape[1], x["tail"].shape[2]).numel()
    assert need > 0
    got = call(pool, x, scratch=torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda"))      # NaN in every word
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    room = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    small = call(pool, x, scratch=room[:need - 16])
    check(pool, x, small)
    assert (room == 255).all()
    whole = call(pool, x, scratch=NO_SCRATCH.cuda())
    assert torch.equal(small[0], whole[0]) and torch.equal(small[1], whole[1])


@pytest.mark.parametrize("fmt", [dict(T=1, fp8=True), dict(T=1, B=16, fp8=True), dict(T=1, bits=4, fp8=True), dict(T=3, B=128, fp8=True)], ids=name)
@pytest.mark.parametrize("g,m", [(1, 2), (6, 4), (3, 30)])
def test_scales_and_ids_at_odd_addresses(fmt, g, m):
    pool = Pool(2, 3, 65, K=30, seed=42, **fmt)
    x = make(pool, 1, g, m, [170], [8], [m], seed=43)
    want = call(pool, x)

    def odd(t):
        room = torch.zeros(t.numel() + 1, dtype=torch.uint8, device="cuda")[1:]
        return room.copy_(t.flatten()).view(t.shape)

    sides = []
    for lo in (0, 1):
        e = pool.encoded(lo, lo + 1)
        sides.append(B.Encoded(e.centroids, odd(e.ids), e.codes, odd(e.scales), e.chunk_len, e.n_smooth))
    tail = x["tail"].cuda()
    got = B.attn_tree(x["q"].cuda(), *sides, x["table"].cuda(), ints(x["kv"]), x["k_new"].cuda(), x["v_new"].cuda(), tail_k=tail[:, :1],
                      tail_v=tail[:, 1:], tail_len=ints(x["tails"]), n_nodes=ints(x["nodes"]), mask=bits_of(x["see"]).cuda(), want_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check(pool, x, got)


@pytest.mark.parametrize("g,m,rope", [(1, 6, False), (1, 6, True), (3, 9, False), (4, 12, True), (5, 30, False)])
def test_queries_behind_a_tree_may_hold_anything(g, m, rope):
    pool = Pool(2, 4, 60, K=16, T=2, seed=44)
    x = make(pool, 1, g, m, [200, 90], [7, 0], [m - 2, 1], seed=45, rope=rope)
    want = call(pool, x)
    for b, live in enumerate(x["nodes"]):
        x["q"][b, :, live:] = float("nan")
        x["k_new"][b, :, live:] = float("nan")
        x["v_new"][b, :, live:] = float("inf")
    got = call(pool, x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("g,m,rope", [(1, 7, False), (3, 8, False), (6, 12, True), (9, 16, False)])
def test_rows_that_see_only_some_or_nothing(g, m, rope):
    """No page, no tail: a mask with empty rows, rows that see one token that is not their own, and bits behind the last node."""
    pool = Pool(2, 1, 32, K=4, T=1, seed=46)
    x = make(pool, 1, g, m, [0], [0], [m], seed=47, rope=rope)
    see = torch.zeros(1, m, m, dtype=torch.bool)
    see[0, 2, 0] = see[0, 4, m - 1] = True
    see[0, m - 1] = True
    x["see"] = see
    check(pool, x, call(pool, x))
    words = bits_of(see) | ~((1 << (m % 32)) - 1)          # what lies behind the last node is not looked at
    got = B.attn_tree(x["q"].cuda(), pool.encoded(0, 1), pool.encoded(1, 2), None, None, x["k_new"].cuda(), x["v_new"].cuda(),
                      mask=words.cuda(), want_lse=True)
    check(pool, x, got)


@pytest.mark.parametrize("rows,rope", [((2, 3), False), ((3, 8), True), ((6, 12), True), ((5, 30), False)])
def test_two_graphs_share_a_scratch_and_take_turns(rows, rope):
    g, m = rows
    pool = Pool(2, 6, 200, K=24, T=2, seed=48)
    calls = []
    scratch = None
    for seed, kv in ((49, [1150, 40]), (50, [3, 1200])):
        x = make(pool, 1, g, m, kv, [12, 0], [m, m], seed=seed, rope=rope, R=15)
        x["table"] = torch.stack([torch.randperm(6, generator=torch.Generator().manual_seed(seed)) for _ in range(2)]).to(torch.int32)
        tail = x["tail"].cuda()
        args = (x["q"].cuda(), pool.encoded(0, 1), pool.encoded(1, 2), x["table"].cuda(), ints(kv), x["k_new"].cuda(), x["v_new"].cuda())
        kw = dict(tail_k=tail[:, :1], tail_v=tail[:, 1:], tail_len=ints(x["tails"]), mask=bits_of(x["see"]).cuda(), want_lse=True,
                  k_rope=None if x["rope"] is None else x["rope"].cuda())
        if scratch is None:
            scratch = B.attn_tree_scratch(args[1], 2, g, m, 6, 15)
        want = B.attn_tree(*args, **kw)
        check(pool, x, want)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = B.attn_tree(*args, **kw, scratch=scratch)
        calls.append((graph, got, want, (args, kw)))       # (the graph reads the inputs where they are)
    for turn in range(6):
        graph, got, want, _ = calls[turn % 2]
        got[0].fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_result_in_place_of_the_queries():
    """out may be q: a row is written when all of its block have been read."""
    pool = Pool(2, 6, 100, K=16, T=1, fp8=True, seed=51)
    for g, m in ((1, 4), (3, 10), (4, 40)):
        x = make(pool, 1, g, m, [560], [12], [m], seed=52)
        want = call(pool, x, scratch=NO_SCRATCH.cuda())
        q = x["q"].transpose(1, 2).contiguous().cuda().transpose(1, 2)
        tail = x["tail"].cuda()
        B.attn_tree(q, pool.encoded(0, 1), pool.encoded(1, 2), x["table"].cuda(), ints(x["kv"]), x["k_new"].cuda(), x["v_new"].cuda(),
                    tail_k=tail[:, :1], tail_v=tail[:, 1:], tail_len=ints(x["tails"]), mask=bits_of(x["see"]).cuda(), out=q,
                    scratch=NO_SCRATCH.cuda())
        assert torch.equal(q, want[0])


def test_masks_kept_tokens_and_copies_on_another_stream_and_in_a_graph():
    """A step's three small operators in one graph, replayed with other contents; the tail's lengths are updated in place."""
    n, H, m, path, R = 3, 2, 40, 6, 50
    pool = Pool(4, 5, 33, K=12, T=1, fp8=True, B=16, seed=53)
    e, into = pool.encoded(0, 4), B.alloc_cache(4, 5 * 33, 33, 12, 16, 1, scale_format=B.SCALE_E4M3)
    gen = torch.Generator().manual_seed(54)
    k, v = (torch.randn(n, H, m, D, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    tail = torch.zeros(n, 2 * H, R, D, dtype=torch.bfloat16, device="cuda")
    parents, nodes = random_parents(n, m, 55).cuda(), ints([m, 7, 0])
    take, keep, lens = torch.randint(0, m, (n, path), generator=gen).to(torch.int32).cuda(), ints([6, 0, 3]), ints([0, 5, 9])
    mask, depth = (torch.empty(n, m, 2, dtype=torch.int32, device="cuda"), torch.empty(n, m, dtype=torch.int32, device="cuda"))

    def step():
        B.tree_mask(parents, nodes, mask=mask, depth=depth)
        B.keep_nodes(k, v, take, keep, tail[:, :H], tail[:, H:], lens, out_len=lens)
        B.copy_pages(e, [4, 0, 1], [0, 1, 3], into=into)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    at = torch.tensor([0, 5, 9])
    want_tail = torch.zeros(n, 2 * H, R, D, dtype=torch.bfloat16)

    def expect():
        see, deep = plain_mask(parents.cpu(), nodes.cpu())
        assert torch.equal(mask.cpu(), bits_of(see)) and torch.equal(depth.cpu(), deep)
        for b, count in enumerate(keep.tolist()):
            for i in range(count):
                want_tail[b, :H, at[b]], want_tail[b, H:, at[b]] = k[b, :, take[b, i]].cpu(), v[b, :, take[b, i]].cpu()
                at[b] += 1
        assert torch.equal(lens.cpu().long(), at) and torch.equal(tail.cpu(), want_tail)
        for s, d in ((4, 0), (0, 1), (1, 3)):
            assert torch.equal(into.codes[:, d * 33:d * 33 + 33], e.codes[:, s * 33:s * 33 + 33])
            assert torch.equal(into.scales[:, d * 33:d * 33 + 33], e.scales[:, s * 33:s * 33 + 33])
            assert torch.equal(into.ids[:, d * 33:d * 33 + 33], e.ids[:, s * 33:s * 33 + 33])
            assert torch.equal(into.centroids[:, d], e.centroids[:, s])

    expect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (56, 57, 58):
        parents.copy_(random_parents(n, m, seed))
        keep.copy_(ints([seed % 5, 2, 1]))
        for t in (into.codes, into.scales, into.ids, into.centroids):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        expect()


def test_refusals_that_need_tensors_of_the_gpu():
    pool = Pool(4, 3, 32, K=8, T=1, seed=60)
    e, half = pool.encoded(0, 4), pool.encoded(0, 2)
    q = torch.zeros(1, 2, 1, D, dtype=torch.bfloat16, device="cuda")
    for src, dst in (([3], [0]), ([0], [3]), ([-1], [0]), ([0], [0]), ([0, 1], [2, 2]), ([0, 1], [1, 2])):
        with pytest.raises(B.QvgError):
            B.copy_pages(e, src, dst)
    with pytest.raises(OverflowError):                     # not page 0
        B.copy_pages(e, [1 << 32], [1])
    with pytest.raises(ValueError):
        B.copy_pages(e, [0], [1], into=half)               # fewer units
    narrow = B.Encoded(half.centroids[..., :64].contiguous(), half.ids, half.codes, half.scales, 32)
    short = B.Encoded(half.centroids[:, :2].contiguous(), half.ids, half.codes, half.scales, 32)
    for bad in (narrow, short):
        with pytest.raises(ValueError):
            B.attn_tree(q, bad, bad, None, None, q, q)
    with pytest.raises(ValueError):                        # a V pool of another page length
        B.attn_tree(q, half, B.Encoded(half.centroids, half.ids, half.codes, half.scales, 16), None, None, q, q)
    with pytest.raises(ValueError):                        # three query heads to two KV heads
        B.attn_tree(torch.zeros(1, 3, 1, D, dtype=torch.bfloat16, device="cuda"), half, half, None, None, q, q)
    with pytest.raises(ValueError):                        # K and V of other strides
        B.attn_tree(q, half, half, None, None, q.expand(1, 2, 1, D).clone(), torch.zeros(1, 2, 1, 2 * D, dtype=torch.bfloat16, device="cuda")[..., ::2])
    init = torch.zeros(2, 8, D, dtype=torch.bfloat16, device="cuda")
    cache = B.PagedCache(1, 2, 3, 32, 2, 4, 8, 64, 1, init)
    s = cache.open()
    for bad in (torch.zeros(1, 5, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 5, 64, dtype=torch.bfloat16, device="cuda")):
        with pytest.raises(ValueError):
            cache.append(s, bad)
    with pytest.raises(TypeError):
        cache.append(s, torch.zeros(2, 5, D, device="cuda"))
    assert cache.length(s) == 0


@pytest.mark.parametrize("fmt", [dict(T=2), dict(T=1, B=16, S=4, fp8=True), dict(T=8, B=128)], ids=name)
@pytest.mark.parametrize("g,m,rope", [(1, 3, False), (2, 9, False), (3, 15, True), (4, 40, False)])
@pytest.mark.parametrize("q,scale", [(2.0 ** -126, 1e-3), (2.0 ** -133, 0.1), (2.0 ** -133, 1e-6), (0.0, 0.1), (1.0, 1e-38)])
def test_queries_so_small_that_all_scores_are_zero(fmt, g, m, rope, q, scale):
    """The row's scale leaves fp32's range; hidden tokens stay hidden, all others count alike."""
    pool = Pool(2, 3, 50, K=12, seed=61, **fmt)
    x = make(pool, 1, g, m, [110, 20], [5, 0], [m, 2], seed=62, rope=rope)
    x["q"] = (torch.sign(x["q"].float()) * q).to(torch.bfloat16)
    check(pool, x, call(pool, x, softmax_scale=scale), scale=scale)


def test_a_scratch_that_is_no_plain_memory_is_refused():
    pool = Pool(2, 6, 200, K=16, T=2, seed=63)
    x = make(pool, 1, 1, 2, [1100], [9], [2], seed=64)
    for bad in (torch.empty(1 << 21, dtype=torch.uint8, device="cuda")[::2], torch.empty(1 << 20, dtype=torch.float32, device="cuda"),
                torch.empty(1 << 20, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            call(pool, x, scratch=bad)
