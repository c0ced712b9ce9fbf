"""Divided attention over 16-bit pages in its forms: every case says whether its call is divided (a call that is not would compare the
undivided form with itself), and that nothing behind the scratch is written."""
import pytest
import torch

from paper_2602_02958_amd import binding as B
from rows_util import check_attention
from test_gpu_attn_pages import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F16 = torch.bfloat16, torch.float16


def check(c, tiles, divided=True):
    """c over tables of at least `tiles` tiles of 32 tokens (entries behind a sequence's pages are not looked at)."""
    n, L = len(c.kv), c.k.shape[2]
    per_page = -(-L // 32) if L % 32 == 0 or L >= 256 else L / 32
    more = max(0, int(tiles / per_page) + 2 - c.table.shape[1])
    c.table = torch.cat([c.table, torch.full((n, more), -(1 << 31), dtype=torch.int32)], 1)
    want, args = c.want(), c.device()
    group, m = c.q.shape[1] // c.k.shape[0], c.q.shape[2]
    need = B._pages_scratch_bytes(n, c.k.shape[0], c.k.shape[3], group, m, c.table.shape[1], L, 0 if c.window is None else min(c.window, 0x7fffffff), c.sink)
    assert (need > 0) == divided
    room = torch.full((need + 4096,), 173, dtype=torch.uint8, device=DEV)
    for scratch in (room[:need], torch.empty(0, dtype=torch.uint8, device=DEV)):
        out, lse = B.attn_pages(**args, want_lse=True, scratch=scratch)
        check_attention(out, lse, want)
    assert (room[need:] == 173).all()
    return args, room[:need]


def lengths(n, long, usual):
    """{sequence: tokens} among n of usual(i) tokens."""
    return [long.get(i, usual(i)) for i in range(n)]


# More sequences than the chip has workgroups for twice: the extra slots go to those that are much longer
@pytest.mark.parametrize("d,dtype,L", [(64, BF, 32), (128, F16, 64), (128, BF, 48)])
def test_one_long_sequence_among_many(d, dtype, L):
    """n > extra: the share stays, usual sequences leave no partial results."""
    check(Case(lengths(70, {13: 2500}, lambda i: 40 + i), None, H=8, g=1, d=d, L=L, dtype=dtype, seed=1), 290)


def test_long_sequences_in_several_groups_of_64():
    kv = lengths(256, {0: 1100, 63: 350, 64: 1200, 130: 0, 191: 700, 255: 1199}, lambda i: (i * 37) % 40)
    check(Case(kv, None, H=4, g=2, d=64, L=32, seed=2), 290)                       # n > extra (128)
    check(Case(kv, None, H=2, g=1, d=64, L=100, dtype=F16, seed=3), 300)           # n = extra (256)


def test_more_extra_slots_than_sequences():
    """n < extra though no sequence gets two: the share is halved."""
    kv = lengths(100, {7: 2400, 70: 1500, 99: 2400}, lambda i: (i * 53) % 100)
    check(Case(kv, None, H=4, g=1, d=64, L=64, seed=4), 270)
    check(Case(kv, None, H=4, g=1, d=64, L=64, seed=5, window=3000, sink=70), 270, divided=False)      # (less than 256 tiles are seen)
    check(Case([min(x, 1500) for x in kv[:60]], None, H=3, g=1, d=256, L=256, seed=6), 270)


@pytest.mark.parametrize("kv", [[300] * 70, [0] * 70, [0] * 69 + [2000], [2000] + [0] * 69, [1] * 70], ids=["equal", "empty", "last", "first", "single"])
def test_batches_that_leave_slots_over(kv):
    check(Case(kv, None, H=8, g=1, d=64, L=32, seed=7), 290)


@pytest.mark.parametrize("d,dtype", [(64, F16), (128, BF), (192, BF), (256, F16)])
def test_many_sequences_of_blocks_of_32_rows(d, dtype):
    """Partial results of 32 rows, blocks that are not full, counts of new tokens that differ."""
    kv = lengths(40, {3: 1600, 38: 900}, lambda i: 6 + i)
    check(Case(kv, [5 - i % 3 for i in range(40)], H=4, g=5, m=5, d=d, L=32, dtype=dtype, seed=8), 270)


# At least two workgroups to a sequence
def test_more_than_64_sequences_of_two_slots():
    kv = lengths(200, {5: 900, 66: 600, 140: 800, 199: 1000}, lambda i: (i * 29) % 50)
    check(Case(kv, None, H=1, g=2, d=64, L=32, seed=9), 64)
    check(Case(kv, [1 + i % 2 for i in range(200)], H=1, g=1, m=2, d=128, L=50, dtype=F16, seed=10), 64)


@pytest.mark.parametrize("d,dtype,g,m,L", [(64, BF, 4, 6, 48), (96, F16, 17, 1, 100), (128, BF, 3, 40, 7), (192, F16, 1, 33, 31), (256, BF, 16, 2, 250)])
@pytest.mark.parametrize("kv", [[2000], [1500, 17, 1000]], ids=["one", "three"])
def test_blocks_of_32_rows_over_pages_that_end_inside_tiles(d, dtype, g, m, L, kv):
    check(Case(kv, None, H=2, g=g, m=m, d=d, L=L, dtype=dtype, seed=11), 40)


@pytest.mark.parametrize("window,sink", [(1000, 0), (1500, 90), (1 << 33, 0)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("L", [32, 100, 257])
def test_windows_of_divided_calls(window, sink, causal, L):
    check(Case([2500, 1800, 30, 0], [4, 1, 4, 4], H=2, g=3, m=4, d=64, L=L, window=window, sink=sink, causal=causal, seed=12), 60)


def test_equal_calls_give_equal_bits_whatever_the_scratch_held():
    args, scratch = check(Case(lengths(70, {13: 2500}, lambda i: 40 + i), None, H=8, g=1, d=64, L=32, seed=13), 290)
    first = B.attn_pages(**args, scratch=scratch)
    for fill in (0, 255):
        scratch.fill_(fill)
        assert torch.equal(B.attn_pages(**args, scratch=scratch), first)
    # less scratch than the call needs: undivided, and nothing is written
    scratch.fill_(99)
    B.attn_pages(**args, scratch=scratch[:-16])
    assert (scratch == 99).all()
