"""What a paged cache of keys from before the rotary embedding asks of the table that turns them (no GPU)."""
import pytest
import torch

from paper_2602_02958_amd import binding as B


@pytest.fixture
def turns(monkeypatch):
    """rope on the host, which keys it was given."""
    monkeypatch.setattr(B, "_check", lambda *a: None)
    monkeypatch.setattr(B, "_here", lambda *a: None)
    seen = []

    def rope(x, table, first=None):
        seen.append((x.shape[2], int(first)))
        return x + 1
    monkeypatch.setattr(B, "rope", rope)
    return seen


def cache():
    init = torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    return B.PagedCache(1, 2, 6, 8, 4, 20, 8, 64, 1, init, device="cpu", pre_rope=True)


def tokens(n):
    return torch.randn(2, n, 128).to(torch.bfloat16)


def test_a_table_without_the_new_tokens_places_is_refused(turns):
    """Beyond a table the nearest row counts, so that a short one would turn keys by a place that is not theirs."""
    c, table = cache(), torch.zeros(7, 64, 2, dtype=torch.float16)
    s = c.open()
    c.append(s, tokens(4), k_rope=table)
    for n in (4, 30):
        with pytest.raises(ValueError, match="places"):
            c.append(s, tokens(n), k_rope=table)
    assert c.length(s) == 4 and turns == [(4, 0)]
    c.append(s, tokens(3), k_rope=table)
    assert c.length(s) == 7 and turns == [(4, 0), (3, 4)]


def test_a_call_that_the_pool_has_no_room_for_turns_nothing(turns):
    c = cache()
    s = c.open()
    with pytest.raises(ValueError, match="pages"):
        c.append(s, tokens(100), k_rope=torch.zeros(200, 64, 2, dtype=torch.float16))
    assert turns == [] and c.length(s) == 0
