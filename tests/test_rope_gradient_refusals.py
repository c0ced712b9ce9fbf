"""What rope refuses of calls that a gradient is recorded of (no GPU: every call ends before the library's)."""
import pytest
import torch

from paper_2602_02958_amd import binding as B


@pytest.fixture
def calls(monkeypatch):
    """What went on to the library."""
    seen = []
    monkeypatch.setattr(B, "_rope", lambda x, *a: seen.append(a) or x.clone())
    return seen


def args():
    return torch.zeros(1, 2, 3, 16), torch.zeros(9, 8, 2)


def test_a_gradient_that_would_be_lost_is_refused(calls):
    x, t = args()
    with pytest.raises(ValueError, match="out"):
        B.rope(x.requires_grad_(), t, out=torch.empty(1, 2, 3, 16))
    with pytest.raises(ValueError, match="out"):
        B.rope(x, t, out=x)
    with pytest.raises(ValueError, match="table"):
        B.rope(x.detach(), t.requires_grad_())
    with pytest.raises(ValueError, match="table"):
        B.rope(x, t)
    assert not calls
    with torch.no_grad():                                    # (nothing is recorded)
        assert not B.rope(x, t, out=x).requires_grad
    assert len(calls) == 1


def test_a_gradient_is_the_turn_back_by_the_places_of_the_call(calls):
    x, t = args()
    first = torch.tensor([4], dtype=torch.int32)
    y = B.rope(x.requires_grad_(), t, first=first, half=True)
    assert y.requires_grad and calls[0][2].tolist() == [4] and calls[0][3:5] == (True, False)
    first += 3                                               # (a step's lengths move on)
    y.sum().backward()
    assert len(calls) == 2 and calls[1][0] is t and calls[1][2].tolist() == [4] and calls[1][3:5] == (True, True)
    assert x.grad.shape == x.shape


def test_a_table_that_was_written_since_is_an_error(calls):
    x, t = args()
    y = B.rope(x.requires_grad_(), t)
    t.zero_()
    with pytest.raises(RuntimeError, match="modified"):
        y.sum().backward()
