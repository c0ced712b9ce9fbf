"""Vector registers that the kernels of rotary positions and 16-bit pages spill, read from the built library's own kernel descriptors (no GPU): none,
but a few of the attention's 256 channels by blocks of 32 rows, whose 512 registers are all in use.  The bounds are the counts of the library
when its times were taken."""
import itertools

import pytest

from test_kernel_registers import spilled  # noqa: F401

SPILLS = {("PgBf16", 256, 2, True): 10, ("PgBf16", 256, 2, False): 8, ("PgF16", 256, 2, True): 12}      # type, channels, blocks of 16 rows, paged


@pytest.mark.parametrize("kind", ["PgBf16", "PgF16"])
@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
def test_attention_over_16_bit_pages(spilled, d, kind):  # noqa: F811
    forms = [(rb, paged, once) for rb, paged, once in itertools.product((1, 2), (False, True), (False, True)) if rb == 2 or once]
    for rb, paged, once in forms:
        name = f"attn_pages_kernel<qvg::{kind}, {d}, {rb}, {str(paged).lower()}, {str(once).lower()}>"
        assert spilled[name] <= SPILLS.get((kind, d, rb, paged), 0), name
    mine = [n for n in spilled if n.startswith(f"attn_pages_kernel<qvg::{kind}, {d},")]
    assert len(mine) == len(forms)                           # (no form that no call reaches)
    joins = [n for n in spilled if n.startswith(f"join_pages_kernel<qvg::{kind}, {d},")]
    assert sorted(joins) == sorted(f"join_pages_kernel<qvg::{kind}, {d}, {per}>" for per in (2, 1024 // d)) and not any(spilled[n] for n in joins)


def test_tables_and_rows(spilled):  # noqa: F811
    mine = [n for n in spilled if n.startswith(("rope_table_kernel", "turn_kernel", "append_lengths_kernel"))]
    assert len(mine) > 60 and not any(spilled[n] for n in mine)
