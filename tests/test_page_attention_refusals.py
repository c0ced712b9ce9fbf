"""Attention over 16-bit pages into its own queries: refused on the CPU (every call fails before any launch), allowed on the GPU."""
import pytest
import torch

from paper_2602_02958_amd import binding as B
from test_rows_refusals import BAD, attend, step


@pytest.mark.parametrize("other", [dict(out_stride_seq=1536), dict(out_stride_head=256), dict(out_stride_token=256, n_new=2)])
def test_out_is_q_with_the_same_strides_only(other):
    """Rows of other places would be written before they are read."""
    t = step(**other)
    t.out = t.q
    assert attend(t=t) == BAD


@pytest.mark.gpu
def test_strides_of_one_element_say_nothing():
    k, v = (torch.randn(2, 3, 16, 64, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in (1, 2))
    q = torch.randn(1, 4, 1, 64, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    table, kv = torch.tensor([[2, 0]], dtype=torch.int32, device="cuda"), torch.tensor([20], dtype=torch.int32, device="cuda")
    want = B.attn_pages(q, k, v, table, kv)
    same = q.as_strided((1, 4, 1, 64), (8192, 64, 4096, 1))
    B.attn_pages(q, k, v, table, kv, out=same)
    assert torch.equal(q, want)
