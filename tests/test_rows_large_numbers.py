"""Numbers beyond the C interface's 32 and 64 bits are refused, not cut to their low bits (no GPU: every call fails before any launch)."""
import pytest
import torch

from paper_2602_02958_amd import binding as B
from test_rows_refusals import BAD, args


@pytest.fixture(autouse=True)
def device_zero(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(B, "_stream", lambda: None)


@pytest.mark.parametrize("first", [-1, -(1 << 64), 1 << 31, 1 << 64, (1 << 64) + 5])
def test_first_places_of_a_table(first):
    a = args()
    with pytest.raises(B.QvgError) as e:
        B.rope_table(9, a["freq"], first=first, out=a["table"])
    assert e.value.status == BAD


@pytest.mark.parametrize("sink", [-1, -(1 << 32), -(1 << 32) + 3])
def test_first_tokens_of_a_window(sink):
    a = args()
    with pytest.raises(B.QvgError) as e:
        B.attn_pages(a["x"], a["k_pages"], a["v_pages"], a["page_table"], a["kv_len"], window=4, sink=sink, out=a["out"])
    assert e.value.status == BAD
