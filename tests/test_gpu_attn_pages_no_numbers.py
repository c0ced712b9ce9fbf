"""Rows of an attention over 16-bit pages whose scores are no numbers: they say so (the lse at least), and no other row does."""
import math

import pytest
import torch

from paper_2602_02958_amd import binding as B
from test_gpu_attn_pages import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"


def both(args):
    """Divided and undivided."""
    return [B.attn_pages(**args, want_lse=True, scratch=scratch) for scratch in (None, torch.empty(0, dtype=torch.uint8, device=DEV))]


@pytest.mark.parametrize("d,dtype,g,m,kv,divided", [(128, torch.bfloat16, 2, 3, [3000, 40], True), (64, torch.float16, 1, 1, [2000], True),
                                                    (256, torch.bfloat16, 3, 20, [700, 90], False), (192, torch.float16, 8, 9, [5000], True)])
def test_queries_that_are_no_numbers(d, dtype, g, m, kv, divided):
    c = Case(kv, [max(1, m - 1)] * len(kv), H=2, g=g, m=m, d=d, L=32, dtype=dtype, seed=1)
    args = c.device()
    need = B.attn_pages_scratch(args["k_pages"], len(kv), g, m, c.table.shape[1]).numel()
    assert (need > 0) == divided
    clean = both(args)
    hit = torch.zeros(c.q.shape[:3], dtype=torch.bool)
    hit[0, 0, 0] = hit[-1, 2 * g - 1, max(1, m - 1) - 1] = hit[0, g, m // 2] = True
    args["q"][hit.to(DEV), 5] = math.nan
    args["q"][0, 0, 0] = math.inf
    live = (torch.arange(m) < max(1, m - 1)).expand_as(hit)
    args["q"][~live.to(DEV)] = math.nan                      # rows that are not there may hold anything
    for (out, lse), (want, want_lse) in zip(both(args), clean):
        out, lse, want, want_lse, bad = out.cpu(), lse.cpu(), want.cpu(), want_lse.cpu(), hit & live
        assert out[bad].isnan().all() and lse[bad].isnan().all()
        assert torch.equal(out[~bad], want[~bad]) and torch.equal(lse[~bad], want_lse[~bad])
        assert (out[~live] == 0).all() and (lse[~live] == -math.inf).all()


def test_a_score_that_overflows_and_rows_that_do_not_see_it():
    """Token 50's key is infinite along the first channel: rows from place 50 on that turn to it have no number, those before it, those whose
    window is past it and those that turn away are as without it."""
    c = Case([70], [40], H=1, g=1, m=40, d=64, L=16, window=12, seed=2, poison=False)
    c.k[0, c.table[0, 50 // 16], 50 % 16, 0] = 0.0
    c.q[..., 0] = torch.where(torch.arange(40) % 3 == 0, -1.0, 1.0).to(c.q.dtype)
    want, want_lse = both(c.device())[1]
    c.k[0, c.table[0, 50 // 16], 50 % 16, 0] = math.inf
    for out, lse in both(c.device()):
        for i in range(40):
            place = 30 + i
            sees = place >= 50 > place - 12
            if sees and i % 3:
                assert out[0, 0, i].isnan().all() and lse[0, 0, i].isnan()
            elif not sees:
                assert torch.equal(out[0, 0, i], want[0, 0, i]) and torch.equal(lse[0, 0, i], want_lse[0, 0, i])
            else:
                assert torch.isfinite(out[0, 0, i].float()).all() and torch.isfinite(lse[0, 0, i])


def test_a_key_that_is_no_number():
    """Only rows that see it lose their lse."""
    c = Case([70], [40], H=1, g=1, m=40, d=64, L=16, window=12, seed=4, poison=False)
    want, want_lse = both(c.device())[1]
    c.k[0, c.table[0, 50 // 16], 50 % 16, 9] = math.nan
    for out, lse in both(c.device()):
        for i in range(40):
            if 30 + i >= 50 > 30 + i - 12:
                assert lse[0, 0, i].isnan()
            else:
                assert torch.equal(out[0, 0, i], want[0, 0, i]) and torch.equal(lse[0, 0, i], want_lse[0, 0, i])


def test_a_row_without_a_number_is_not_left_out_of_a_merge():
    c = Case([200], None, H=1, g=2, d=128, L=16, seed=3)
    args = c.device()
    args["q"][0, 1, 0, 7] = math.nan
    a, la = B.attn_pages(**args, want_lse=True)
    b, lb = torch.ones(2, 1, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 1, device=DEV)
    out, lse = B.attn_merge(a[0].contiguous(), la[0].contiguous(), b, lb, want_lse=True)
    assert torch.isfinite(out[0].float()).all() and out[1].isnan().all() and lse[1].isnan().all()
