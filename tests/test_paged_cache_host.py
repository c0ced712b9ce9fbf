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
