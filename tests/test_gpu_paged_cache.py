"""Tree masks, kept tokens, page copies and the paged cache that uses them together."""
import pytest
import torch

from tree_util import D, Pool, bits_of, plain_mask, random_parents

pytestmark = pytest.mark.gpu
B = pytest.importorskip("paper_2602_02958_amd.binding")


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("seqs,nodes", [(1, 1), (3, 2), (2, 31), (2, 32), (1, 33), (4, 64), (2, 65), (1, 257), (2, 1000), (1, 1024)])
def test_tree_mask(seqs, nodes):
    par = random_parents(seqs, nodes, seqs * 1000 + nodes)
    live = [max(0, nodes - 3 * b) for b in range(seqs)]
    see, depth = plain_mask(par, live)
    m, d = B.tree_mask(par.cuda(), n_nodes=ints(live))
    assert torch.equal(m.cpu(), bits_of(see)) and torch.equal(d.cpu(), depth)


@pytest.mark.parametrize("nodes", [5, 40, 200])
def test_tree_mask_shapes_of_trees(nodes):
    """A chain, a bush, nodes far from their parents, and holes of every kind."""
    i = torch.arange(nodes)
    g = torch.Generator().manual_seed(nodes)
    far = torch.where(i > 0, (torch.rand(nodes, generator=g) * i).long(), -1)
    holes = far.clone()
    holes[nodes // 3], holes[nodes // 2], holes[1] = -2, nodes // 2, nodes + 5
    holes[nodes - 1] = -(1 << 31)
    par = torch.stack([i - 1, torch.full_like(i, -1), torch.zeros_like(i) - (i == 0).long(), far, holes]).to(torch.int32)
    see, depth = plain_mask(par)
    m, d = B.tree_mask(par.cuda())
    assert torch.equal(m.cpu(), bits_of(see)) and torch.equal(d.cpu(), depth)


@pytest.mark.parametrize("seqs,heads,nodes,path", [(1, 1, 1, 1), (3, 2, 9, 5), (2, 5, 64, 33), (2, 3, 4, 4)])
def test_keep_nodes(seqs, heads, nodes, path):
    g = torch.Generator().manual_seed(nodes)
    k, v = (torch.randn(seqs, nodes, heads, D, generator=g).to(torch.bfloat16).cuda().transpose(1, 2) for _ in range(2))
    tail = torch.randn(seqs, 2 * heads, 40, D, generator=g).to(torch.bfloat16).cuda()
    idx = torch.randint(0, nodes, (seqs, path), generator=g).to(torch.int32)          # (an index may come twice)
    idx[0, path - 1] = nodes                                # outside: its row stays
    keep = [path + 3] + [max(0, path - b) for b in range(1, seqs)]
    lens = [38 - 2 * b for b in range(seqs)]                # the first tail runs over
    want = tail.clone()
    for b in range(seqs):
        for i in range(min(path, keep[b])):
            if lens[b] + i < 40 and 0 <= idx[b, i] < nodes:
                want[b, :heads, lens[b] + i] = k[b, :, idx[b, i]]
                want[b, heads:, lens[b] + i] = v[b, :, idx[b, i]]
    length = ints(lens)
    new = B.keep_nodes(k, v, idx.cuda(), ints(keep), tail[:, :heads], tail[:, heads:], length)
    assert torch.equal(tail, want)
    assert new.tolist() == [min(40, n + min(path, c)) for n, c in zip(lens, keep)]
    again = B.keep_nodes(k, v, idx.cuda(), ints(keep), tail[:, :heads], tail[:, heads:], length, out_len=length)
    assert again is length and length.tolist() == new.tolist() and torch.equal(tail, want)


def arrays(e):
    return e.centroids, e.ids, e.codes, e.scales


def pages_of(e):
    L = e.chunk_len
    return [e.centroids] + [t.view(t.shape[0], -1, L, *t.shape[2:]) for t in arrays(e)[1:]]


@pytest.mark.parametrize("fmt", [dict(T=2), dict(T=1, fp8=True), dict(T=3, B=16, S=4, fp8=True, K=7), dict(K=300, T=1, bits=4)],
                         ids=lambda f: "-".join(f"{k}{v}" for k, v in f.items()))
@pytest.mark.parametrize("page", [1, 3, 40, 1000])
def test_copy_pages(fmt, page):
    pool = Pool(3, 7, page, seed=1, **fmt)
    e, other = pool.encoded(0, 3), Pool(3, 9, page, seed=2, **fmt).encoded(0, 3)
    want = [t.clone() for t in pages_of(e)]
    src, dst = [6, 0, 2, 6], [1, 3, 4, 5]                   # a source may be copied twice
    for t in want:
        t[:, dst] = t[:, src]
    assert B.copy_pages(e, src, dst) is e
    for t, w in zip(pages_of(e), want):
        assert torch.equal(t, w)
    want = [t.clone() for t in pages_of(other)]
    for t, s in zip(want, pages_of(e)):
        t[:, [8, 0]] = s[:, [0, 6]]
    B.copy_pages(e, [0, 6], [8, 0], into=other)
    for t, w in zip(pages_of(other), want):
        assert torch.equal(t, w)
    B.copy_pages(e, [], [])


def test_copy_of_more_pages_than_a_launch_takes():
    pool = Pool(1, 450, 2, seed=3)
    e = pool.encoded(0, 1)
    into = B.alloc_cache(1, 450 * 2, 2, 16, 64, 1)
    order = torch.randperm(450, generator=torch.Generator().manual_seed(4)).tolist()
    B.copy_pages(e, order, list(range(450)), into=into)
    for t, w in zip(pages_of(into), pages_of(e)):
        assert torch.equal(t, w[:, order])


def _filled(seed, n, H):
    g = torch.Generator().manual_seed(seed)
    c = torch.randn(2 * H, 12, D, generator=g)
    pick = torch.randint(0, 12, (2 * H, n), generator=g)
    return (torch.gather(c, 1, pick[:, :, None].expand(-1, -1, D)) + 0.2 * torch.randn(2 * H, n, D, generator=g)).to(torch.bfloat16).cuda()


def _cache(H, init, **kw):
    args = dict(heads=H, max_seqs=3, n_pages=9, page_len=64, max_pages=6, max_new=12, n_clusters=16, group_size=64, n_stages=2, init=init)
    args.update(kw)
    return B.PagedCache(**args)


def test_a_rollout_of_steps_forks_and_compactions():
    """Prompts, trees, kept paths, forks, closings and a compaction; the attention stays that of the tokens as they were put in,
    which a second cache per sequence, without sharing or moving, holds as well."""
    H, g, m = 2, 2, 12
    first = _filled(1, 150, H)
    init = first[:, :16].contiguous()
    c = _cache(H, init)
    mirror = [_cache(H, init, max_seqs=1) for _ in range(3)]
    a = c.open()
    c.append(a, first)
    mirror[0].open()
    mirror[0].append(0, first[:, :70])                      # the same tokens in two pieces
    mirror[0].append(0, first[:, 70:])
    assert c.length(a) == 150 and c.pages[a] != [] and c.tails[a] == 150 % 64
    b = c.fork(a)
    mirror[1].open()
    mirror[1].append(0, first)
    assert c.pages[b] == c.pages[a] and c.free_pages() == 7
    gen = torch.Generator().manual_seed(5)
    for step in range(14):
        open_ = [s for s in range(3) if c.pages[s] is not None]
        live = [m if s in open_ else 0 for s in range(3)]
        q = torch.randn(3, m, H * g, D, generator=gen).to(torch.bfloat16).cuda().transpose(1, 2)
        k, v = (torch.randn(3, m, H, D, generator=gen).to(torch.bfloat16).cuda().transpose(1, 2) for _ in range(2))
        par = random_parents(3, m, step)
        mask, depth = B.tree_mask(par.cuda(), n_nodes=ints(live))
        out, lse = c.attend(q, k, v, n_nodes=ints(live), mask=mask, want_lse=True)
        for s in range(3):
            if s not in open_:
                assert (out[s] == 0).all() and torch.isneginf(lse[s]).all()
                continue
            o, z = mirror[s].attend(q[s:s + 1], k[s:s + 1], v[s:s + 1], mask=mask[s:s + 1], want_lse=True)
            # the two differ by how the sums are divided: binary16 weights (2^-11) of values below 8, and the result's rounding
            assert torch.allclose(out[s].float(), o[0].float(), rtol=2.0 ** -7, atol=2.0 ** -11 * 8)
            assert torch.allclose(lse[s], z[0], rtol=0, atol=2.0 ** -10)
        path = torch.zeros(3, 4, dtype=torch.int32)
        counts = [0, 0, 0]
        for s in open_:
            node = int(torch.randint(0, m, (1,), generator=gen))
            way = [j for j in range(m) if plain_mask(par[s:s + 1])[0][0, node, j]][:4]
            path[s, :len(way)] = torch.tensor(way)
            counts[s] = len(way)
        c.keep(k, v, path.cuda(), counts)
        for s in open_:
            mirror[s].keep(k[s:s + 1], v[s:s + 1], path[s:s + 1].cuda(), counts[s:s + 1])
            assert mirror[s].length(0) == c.length(s) and c.tail_len[s].item() == c.tails[s]
        if step == 6:
            c.close(a)
            assert c.compact() == 9 - c.free_pages() and max(c.pages[b]) < 9 - c.free_pages()
        if step == 9:
            d = c.fork(b)
            assert d == 0
            mirror[0] = _cache(H, init, max_seqs=1)
            mirror[0].open()
            mirror[0].pages, mirror[0].tails = [list(range(len(c.pages[d])))], [c.tails[d]]
            for page in mirror[0].pages[0]:
                mirror[0].holders[page] = 1
            c.gather(d, into=mirror[0].pool) if len(c.pages[d]) else None
            mirror[0].tail[0].copy_(c.tail[d])
            mirror[0]._tell(0)
    # the pages, gathered, are the cache that the other entry points read
    e = c.gather(b)
    n = len(c.pages[b]) * 64
    assert e.ids.shape == (2 * H, n)
    q = torch.randn(H, 5, D, generator=gen).to(torch.bfloat16).cuda()
    side = lambda lo: B.Encoded(e.centroids[lo:lo + H], e.ids[lo:lo + H], e.codes[lo:lo + H], e.scales[lo:lo + H], 64)
    o, z = B.attn_decode(q, side(0), side(H), want_lse=True)
    zero = torch.zeros(1, H, 5, D, dtype=torch.bfloat16, device="cuda")
    kv = ints([n])
    o2, z2 = B.attn_tree(q[None], side(0), side(H), ints([list(range(n // 64))]), kv, zero, zero,
                         mask=torch.zeros(1, 5, 1, dtype=torch.int32, device="cuda"), want_lse=True)
    # (attn_decode rounds the decoded values to bf16 first: 2^-8 of values below 8, and of scores below 16)
    assert torch.allclose(o.float(), o2[0].float(), rtol=2.0 ** -7, atol=2.0 ** -8 * 8)
    assert torch.allclose(z, z2[0], rtol=0, atol=2.0 ** -8 * 16)


def test_the_cache_refuses_what_it_has_no_room_for_and_stays_as_it_was():
    H = 1
    c = _cache(H, _filled(9, 16, H), n_pages=3, max_pages=2)
    s = c.open()
    with pytest.raises(ValueError, match="more than 2 pages"):
        c.append(s, _filled(2, 64 * 3, H))
    c.append(s, _filled(2, 127, H))
    t = c.open()
    c.append(t, _filled(3, 63, H))
    assert (c.length(s), c.length(t), c.free_pages()) == (127, 63, 2)
    k = torch.zeros(3, H, 4, D, dtype=torch.bfloat16, device="cuda")
    path = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    for bad in ([0, 0], [3, 0, 0], [-1, 0, 0]):
        with pytest.raises(ValueError, match="n_keep"):
            c.keep(k, k, path, bad)
    with pytest.raises(ValueError, match="not open"):
        c.keep(k, k, path, [0, 0, 1])
    u = c.open()
    c.append(u, _filled(4, 63, H))
    c.keep(k, k, path, [0, 1, 0])
    c.keep(k, k, path, [0, 0, 0])
    with pytest.raises(ValueError, match="2 pages are needed, 1 are free"):
        c.keep(k, k, path, [1, 0, 1])
    assert (c.length(s), c.length(t), c.length(u)) == (127, 64, 63) and c.tail_len.tolist() == [63, 0, 63]
    with pytest.raises(ValueError, match="all places"):
        c.fork(s)
    c.close(t)
    with pytest.raises(ValueError, match="not open"):
        c.fork(t)
    assert c.free_pages() == 2
