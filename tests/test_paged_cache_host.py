"""What a paged cache does on the host: refusals, and its books."""
import pytest
import torch

from paper_2602_02958_amd import binding as B


def cache(**kw):
    init = torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    args = dict(heads=1, max_seqs=2, n_pages=6, page_len=8, max_pages=4, max_new=20, n_clusters=8, group_size=64, n_stages=1, init=init,
                device="cpu")
    args.update(kw)
    return B.PagedCache(**args)


def test_keys_before_the_rotary_embedding_need_a_cache_of_such_keys():
    """A table rotates what the pages hold, and the tail holds what was attended to: one form in both would be attended to wrongly."""
    x = torch.zeros(2, 1, 3, 128, dtype=torch.bfloat16)
    table, path = torch.zeros(40, 64, 2, dtype=torch.float16), torch.zeros(2, 2, dtype=torch.int32)
    plain, pre = cache(), cache(pre_rope=True)
    with pytest.raises(ValueError, match="k_rope"):
        plain.attend(x, x, x, k_rope=table)
    with pytest.raises(ValueError, match="k_rope"):
        pre.attend(x, x, x)
    with pytest.raises(ValueError, match="k_rotated"):
        plain.keep(x, x, path, [0, 0], k_rotated=x)
    with pytest.raises(ValueError, match="k_rotated"):
        pre.keep(x, x, path, [0, 0])


def test_append_takes_the_rotated_keys_beside_the_stored_ones(monkeypatch):
    monkeypatch.setattr(B, "_check", lambda *a: None)
    monkeypatch.setattr(B, "_here", lambda *a: None)
    kv, rot = torch.randn(2, 5, 128).to(torch.bfloat16), torch.randn(1, 5, 128).to(torch.bfloat16)
    plain, pre = cache(), cache(pre_rope=True)
    s, t = plain.open(), pre.open()
    with pytest.raises(ValueError, match="k_rotated"):
        plain.append(s, kv, k_rotated=rot)
    for bad in (None, rot[:, :4], kv):
        with pytest.raises(ValueError, match="k_rotated"):
            pre.append(t, kv, k_rotated=bad)
    assert pre.length(t) == 0
    pre.append(t, kv, k_rotated=rot)
    assert pre.length(t) == 5 and torch.equal(pre.tail[t, :2, :5], kv) and torch.equal(pre.tail[t, 2:, :5], rot)
    plain.append(s, kv)
    assert plain.tail.shape[1] == 2 and torch.equal(plain.tail[s, :, :5], kv)
    u = pre.fork(t)
    assert torch.equal(pre.tail[u, :, :5], pre.tail[t, :, :5])


class Host:
    """The cache's kernels on the host: pages hold the tokens themselves; the n-th encode fails."""

    def __init__(self, monkeypatch, fail_at):
        self.pages, self.left = {}, fail_at
        monkeypatch.setattr(B, "_check", lambda *a: None)
        monkeypatch.setattr(B, "_here", lambda *a: None)
        monkeypatch.setattr(B, "encode_chunk", self.encode)
        monkeypatch.setattr(B, "keep_nodes", self.keep)

    def encode(self, x, *a, chunk_index, **kw):
        self.left -= 1
        if self.left == 0:
            raise B.QvgError(-6, "qvg_encode_chunk")
        self.pages[chunk_index] = x.clone()

    @staticmethod
    def keep(k_new, v_new, path, n_keep, tail_k, tail_v, tail_len, out_len=None):
        for b, n in enumerate(n_keep.tolist()):
            at = int(tail_len[b])
            tail_k[b, :, at:at + n], tail_v[b, :, at:at + n] = k_new[b, :, path[b, :n].long()], v_new[b, :, path[b, :n].long()]
        out_len.copy_(tail_len + n_keep)

    def tokens(self, c, s):
        """What a sequence holds, as the device's copies of its pages and lengths say."""
        n = int(c.kv_len[s]) // c.page_len
        return torch.cat([self.pages[p] for p in c.table[s, :n].tolist()] + [c.tail[s, :, :int(c.tail_len[s])]], 1)


@pytest.mark.parametrize("fail_at", [1, 2, 3])
@pytest.mark.parametrize("first", [0, 5])
def test_an_append_that_fails_leaves_what_it_has_taken_in(monkeypatch, fail_at, first):
    c, kv = cache(n_pages=12, max_pages=8), torch.randn(2, 60, 128).to(torch.bfloat16)
    host = Host(monkeypatch, fail_at)
    s = c.open()
    c.append(s, kv[:, :first])
    with pytest.raises(B.QvgError):
        c.append(s, kv[:, first:30])
    for _ in range(2):
        n = c.length(s)
        assert n == int(c.kv_len[s]) + int(c.tail_len[s]) and len(c.pages[s]) == int(c.kv_len[s]) // 8 == 12 - c.free_pages()
        assert torch.equal(host.tokens(c, s), kv[:, :n])
        c.append(s, kv[:, n:n + 21])                       # and goes on from there
    assert c.tails[s] < 8


@pytest.mark.parametrize("fail_at", [1, 2, 3, 4])
def test_a_keep_that_fails_while_encoding_has_kept_all(monkeypatch, fail_at):
    """Two sequences with more new tokens than two pages hold: whichever encode fails, no token is lost or comes twice."""
    c = cache(n_pages=12, max_pages=6)
    host = Host(monkeypatch, fail_at)
    kv = torch.randn(2, 2, 50, 128).to(torch.bfloat16)      # [sequence, unit, token]
    path = torch.arange(20, dtype=torch.int32).expand(2, 20).contiguous()
    for s in range(2):
        c.open()
        c.append(s, kv[s, :, :6])

    def keep(at):
        new = kv[:, :, at:at + 20]
        c.keep(new[:, :1], new[:, 1:], path, [20, 20])

    with pytest.raises(B.QvgError):
        keep(6)
    for s in range(2):
        assert c.length(s) == int(c.kv_len[s]) + int(c.tail_len[s]) == 26
        assert torch.equal(host.tokens(c, s), kv[s, :, :26])
    keep(26)
    for s in range(2):
        assert c.length(s) == 46 and c.tails[s] == int(c.tail_len[s]) == 6 and torch.equal(host.tokens(c, s), kv[s, :, :46])


@pytest.mark.parametrize("page_len,group_size,n_stages,fits", [(8, 128, 1, True), (7, 128, 1, False), (4, 64, 1, True), (6, 64, 1, False),
                                                               (2, 64, 2, True), (1, 16, 1, True), (33, 64, 2, False), (33, 32, 2, True)])
def test_pages_whose_scales_would_not_be_aligned_are_refused(page_len, group_size, n_stages, fits):
    """The encoder writes binary16 scales from 16-byte boundaries on: the second page of such a pool could never be written."""
    args = dict(page_len=page_len, group_size=group_size, n_stages=n_stages)
    cache(scale_format=B.SCALE_E4M3, **args)
    if fits:
        c = cache(**args)
        assert c.pool.scales[0, page_len:].data_ptr() % 16 == c.pool.scales.data_ptr() % 16
    else:
        with pytest.raises(ValueError, match="page_len"):
            cache(**args)
