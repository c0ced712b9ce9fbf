"""Views of pages, as the library is told of them (no GPU)."""
import torch

from paper_2602_02958_amd import binding as B


def test_pages_of_one_token_have_no_stride_between_tokens():
    """It says nothing, and may be larger than one that does."""
    table, kv = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for shape, strides in (((2, 5, 1, 64), (320, 64, 1 << 25, 1)), ((2, 5, 1, 64), (320, 64, 64, 1))):
        k, v = (torch.empty(2 * 5 * 64, dtype=torch.bfloat16).as_strided(shape, strides) for _ in range(2))
        for written in (False, True):
            c = B._page_cache(k, v, table, kv, written)
            assert (c.page_len, c.stride_head, c.stride_page, c.stride_token) == (1, 320, 64, 0)
    k, v = B.alloc_pages(2, 5, 4, 64, device="cpu")
    assert B._page_cache(k, v, table, kv).stride_token == 64
