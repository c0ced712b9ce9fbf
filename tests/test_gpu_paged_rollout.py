"""A paged cache over a rollout against the definition: every page is the encoder's output for the tokens that were put in at its
place, and every step's attention is that over those pages and the tail's own tokens in 64 bits (tree_util.reference, which
derives the tolerances)."""
import pytest
import torch

from tree_util import D, Pool, plain_mask, random_parents, reference, rotate

pytestmark = pytest.mark.gpu
B = pytest.importorskip("paper_2602_02958_amd.binding")


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rope_table(n):
    ang = torch.arange(n, dtype=torch.float64)[:, None] * 1000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
    return torch.stack([ang.cos(), ang.sin()], -1).to(torch.float16)


class Sequence:
    """What was put into a sequence: kv [2H, n, D] as stored, rot [H, n, D] the keys as attended to, and the pages that follow."""

    def __init__(self, H):
        self.kv, self.rot, self.pages = torch.zeros(2 * H, 0, D, dtype=torch.bfloat16), torch.zeros(H, 0, D, dtype=torch.bfloat16), []

    def put(self, kv, rot):
        self.kv, self.rot = torch.cat([self.kv, kv], 1), torch.cat([self.rot, rot], 1)

    def copy(self):
        s = Sequence.__new__(Sequence)
        s.kv, s.rot, s.pages = self.kv, self.rot, list(self.pages)
        return s

    def encode(self, cache):
        L = cache.page_len
        while (len(self.pages) + 1) * L <= self.kv.shape[1]:
            i = len(self.pages)
            init = self.pages[-1].centroids[:, 0] if i else cache.init
            p = cache.pool
            self.pages.append(B.encode_chunk(self.kv[:, i * L:(i + 1) * L].cuda(), init, cache.group_size, cache.n_stages,
                                             cache.warm_iters if i else cache.cold_iters, bits=p.bits, scale_format=p.scale_format))
        return self.pages


def stored_pool(pages, like: Pool):
    """The pages, one behind the other, as tree_util.Pool decodes them (its stored values are not its own draw)."""
    host = lambda name: torch.cat([getattr(p, name).cpu() for p in pages], 1)                              # noqa: E731
    pool = Pool.__new__(Pool)
    pool.L, pool.T, pool.S, pool.B, pool.bits, pool.fp8, pool.pages = like.L, like.T, like.S, like.B, like.bits, like.fp8, len(pages)
    if not pages:
        return pool
    cent, ids, codes, scales = host("centroids"), host("ids").long(), host("codes").long(), host("scales")
    pool.cent = cent if pool.S > 1 else cent[:, :, None]
    pool.ids = ids if pool.S > 1 else ids[:, :, None]
    b = pool.bits
    field = ((codes[..., None] >> (b * torch.arange(8 // b))) & ((1 << b) - 1)).flatten(-2)
    pool.level = torch.where(field >= 1 << (b - 1), field - (1 << b), field)
    if pool.fp8:
        e, m = (scales >> 3).double(), (scales & 7).double()
        pool.scale_values = torch.where(e > 0, (1 + m / 8) * torch.exp2(e - 7), m / 8 * 2.0 ** -6)
    else:
        pool.scale_values = scales.double()
    return pool


def tokens(H, n, seed):
    g = torch.Generator().manual_seed(seed)
    c = torch.randn(2 * H, 12, D, generator=torch.Generator().manual_seed(7))
    pick = torch.randint(0, 12, (2 * H, n), generator=g)
    return (torch.gather(c, 1, pick[:, :, None].expand(-1, -1, D)) + 0.2 * torch.randn(2 * H, n, D, generator=g)).to(torch.bfloat16)


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("fmt,L,m,most", [(dict(T=2), 32, 7, 4), (dict(T=1, B=16, S=4, fp8=True), 32, 7, 4),
                                          (dict(T=1, bits=4, fp8=True), 40, 17, 6), (dict(T=3, B=32), 8, 24, 20), (dict(T=2, fp8=True), 33, 5, 5)],
                         ids=str)
def test_a_rollout_is_the_attention_over_the_tokens_that_were_put_in(fmt, L, m, most, rope):
    H, g, seqs, K = 2, 2, 3, 8
    like = Pool(1, 1, L, K=K, **fmt)
    table = rope_table(400) if rope else None
    turn = lambda k, at: k if table is None else rotate(k.double(), table[at]).to(torch.bfloat16)          # noqa: E731

    first = tokens(H, 64, 1)
    init = first[:, :K * like.S].contiguous().cuda()
    if like.S > 1:
        init = (init.view(2 * H, like.S, K, D).float() * 0.4 ** torch.arange(like.S, device="cuda")[:, None, None]).to(torch.bfloat16)
    c = B.PagedCache(H, seqs, 60, L, 40, m, K, like.B, like.T, init, n_smooth=like.S, bits=like.bits,
                     scale_format=B.SCALE_E4M3 if like.fp8 else B.SCALE_F16, pre_rope=rope)
    held = [None] * seqs

    def put(s, kv):
        n = held[s].kv.shape[1]
        rot = torch.stack([turn(kv[h], torch.arange(n, n + kv.shape[1])) for h in range(H)])
        c.append(s, kv.cuda(), **(dict(k_rotated=rot.cuda()) if rope else {}))
        held[s].put(kv, rot)

    def check_pages(s):
        x = held[s]
        n, pages = x.kv.shape[1], x.encode(c)
        assert c.length(s) == n and len(c.pages[s]) == len(pages) == n // L and c.tails[s] == n % L
        assert c.table[s, :len(pages)].tolist() == c.pages[s]
        assert (c.kv_len[s].item(), c.tail_len[s].item()) == (n // L * L, n % L)
        for page, want in zip(c.pages[s], pages):
            at = slice(page * L, (page + 1) * L)
            assert torch.equal(c.pool.centroids[:, page], want.centroids[:, 0]) and torch.equal(c.pool.ids[:, at], want.ids)
            assert torch.equal(c.pool.codes[:, at], want.codes) and torch.equal(c.pool.scales[:, at], want.scales)

    a = c.open()
    held[a] = Sequence(H)
    put(a, tokens(H, L + 8, 2))
    put(a, tokens(H, L - 3, 3))
    check_pages(a)
    b = c.fork(a)
    held[b] = held[a].copy()
    gen = torch.Generator().manual_seed(11)
    for step in range(12):
        live = [m if held[s] else 0 for s in range(seqs)]
        q = torch.randn(seqs, m, H * g, D, generator=gen).to(torch.bfloat16).transpose(1, 2)
        raw, v = (torch.randn(seqs, m, H, D, generator=gen).to(torch.bfloat16).transpose(1, 2) for _ in range(2))
        par = random_parents(seqs, m, step)
        see, depth = plain_mask(par, live)
        k = torch.empty(seqs, m, H, D, dtype=torch.bfloat16).transpose(1, 2)
        for s in range(seqs):
            at = (held[s].kv.shape[1] if held[s] else 0) + depth[s].clamp(min=0).long()
            for h in range(H):
                k[s, h] = turn(raw[s, h], at)
        dev = [t.transpose(1, 2).contiguous().cuda().transpose(1, 2) for t in (q, k, v, raw)]
        mask, _ = B.tree_mask(par.cuda(), n_nodes=ints(live))
        out, lse = c.attend(dev[0], dev[1], dev[2], n_nodes=ints(live), mask=mask, k_rope=None if table is None else table.cuda(),
                            want_lse=True)
        out, lse = out.double().cpu(), lse.double().cpu()
        path, counts = torch.zeros(seqs, most, dtype=torch.int32), [0] * seqs
        for s in range(seqs):
            if not held[s]:
                assert (out[s] == 0).all() and torch.isneginf(lse[s]).all()
                continue
            x, full = held[s], len(held[s].pages) * L
            tail_k, tail_v, n = x.rot[None, :, full:], x.kv[None, H:, full:], x.kv.shape[1] - full
            want, z, tol, ltol = reference(q[s:s + 1], stored_pool(x.pages, like), H, [list(range(len(x.pages)))], [full], k[s:s + 1],
                                           v[s:s + 1], tail_k, tail_v, [n], [m], see[s:s + 1], table)
            assert ((out[s] - want[0]).abs() <= tol[0] + 1e-30).all() and ((lse[s] - z[0]).abs() <= ltol[0] + 1e-30).all(), (step, s)
            # (as in test_gpu_tree_attn: half a step of bf16 and as much again, over all rows)
            assert (out[s] - want[0]).norm() <= 2.0 ** -7 * want[0].norm(), (step, s)
            node = m - 1 - step % 3
            way = [j for j in range(m) if see[s, node, j]][:most] if most < m // 2 else list(range(m))[:most]
            if most >= m // 2:                             # a chain as long as several pages: the first nodes, at places of a chain
                k[s], at = k[s], x.kv.shape[1] + torch.arange(m)
                for h in range(H):
                    k[s, h] = turn(raw[s, h], at)
            path[s, :len(way)], counts[s] = torch.tensor(way, dtype=torch.int32), len(way)
            x.put(torch.cat([raw[s][:, way], v[s][:, way]]), k[s][:, way])
        rotated = k.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        c.keep(dev[3], dev[2], path.cuda(), counts, **(dict(k_rotated=rotated) if rope else {}))
        for s in range(seqs):
            if held[s]:
                check_pages(s)
        if step == 3:
            put(b, tokens(H, L + 5, 4))
            check_pages(b)
        if step == 5:
            c.close(a)
            held[a] = None
            assert c.compact() == len(c.pages[b]) and sorted(c.pages[b]) == list(range(len(c.pages[b])))
        if step == 8:
            d = c.fork(b)
            held[d] = held[b].copy()
            e = c.open()
            held[e] = Sequence(H)
    assert len(c.pages[b]) >= 3
