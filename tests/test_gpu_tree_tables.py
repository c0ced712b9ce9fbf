"""attn_tree's forms that the lengths of the pages choose: pages long enough for tables of the centroids' scores (three tokens of a page
or more to a centroid for up to 16 query rows, four for more), with tables of every size that the local memory is divided for,
and pools whose pages lie beyond 4 GiB.  Tolerances: tree_util.reference."""
import pytest
import torch

from tree_util import D, Pool, bits_of
from test_gpu_tree_attn import NO_SCRATCH, check, call, ints, make
from test_gpu_tree_forms import PACKED, name

pytestmark = pytest.mark.gpu
B = pytest.importorskip("paper_2602_02958_amd.binding")


@pytest.mark.parametrize("fmt", PACKED, ids=name)
@pytest.mark.parametrize("K,L", [(64, 300), (256, 1040)])
@pytest.mark.parametrize("g,m", [(1, 1), (2, 8), (1, 17), (4, 8), (5, 8)])
def test_tables_of_every_format(fmt, K, L, g, m):
    """1, 16, 17, 32 and 40 rows; the second page is not full and ends inside a tile, a sequence has a page of one token."""
    pool = Pool(2, 3, L, K=K, seed=91, **fmt)
    x = make(pool, 1, g, m, [2 * L - 45, 1], [7, 33], [m, max(1, m - 3)], seed=92)
    check(pool, x, call(pool, x, scratch=NO_SCRATCH.cuda()))


@pytest.mark.parametrize("fmt", [dict(T=1, fp8=True), dict(T=2), dict(T=4), dict(T=3, B=32)], ids=name)
@pytest.mark.parametrize("K", [255, 257, 512])
@pytest.mark.parametrize("g,m", [(1, 1), (1, 16), (2, 12)])
def test_tables_of_words_and_of_odd_sizes(fmt, K, g, m):
    L = 4 * K + 9
    pool = Pool(2, 2, L, K=K, seed=93, **fmt)
    x = make(pool, 1, g, m, [L + 300], [5], [m], seed=94)
    check(pool, x, call(pool, x, scratch=NO_SCRATCH.cuda()))


@pytest.mark.parametrize("fmt", [dict(T=1, B=16, S=4, fp8=True), dict(T=1, B=16, S=4, bits=4, fp8=True)], ids=name)
@pytest.mark.parametrize("K", [16, 255, 256, 512])
@pytest.mark.parametrize("g,m", [(1, 1), (1, 2), (3, 1), (1, 4), (5, 1), (2, 4), (1, 9), (4, 4)])
def test_tables_of_four_stages(fmt, K, g, m):
    """Of as many columns as there are rows, rounded up to a power of two, where sixteen would fill a CU."""
    L = 3 * K + 50
    pool = Pool(2, 2, L, K=K, seed=95, **fmt)
    x = make(pool, 1, g, m, [L + 200], [5], [m], seed=96)
    check(pool, x, call(pool, x, scratch=NO_SCRATCH.cuda()))


@pytest.mark.parametrize("fmt", [dict(T=1, fp8=True), dict(T=2), dict(T=4, B=32), dict(T=1, B=16, S=4, fp8=True)], ids=name)
@pytest.mark.parametrize("g,m", [(1, 1), (2, 10)])
def test_tables_of_a_divided_call(fmt, g, m):
    """Sixteen sequences over sixteen heads that share two pages: as many slots as pages, so that a part meets whole ones."""
    H, L, K = 16, 400, 64
    pool = Pool(2 * H, 2, L, K=K, seed=97, **fmt)
    kv = [2 * L, 2 * L - 30, L + 1] + [40 * b % 97 for b in range(13)]
    x = make(pool, H, g, m, kv, [3] * 16, [m] * 16, seed=98)
    x["table"] = torch.tensor([[0, 1], [1, 0]] * 8, dtype=torch.int32)
    assert B.attn_tree_scratch(pool.encoded(0, H), 16, g, m, 2, x["tail"].shape[2]).numel() > 0
    check(pool, x, call(pool, x))


@pytest.mark.parametrize("spread", [1e-4, 1.0, 30.0])
@pytest.mark.parametrize("qs", [1e-30, 1.0, 1e20])
@pytest.mark.parametrize("fmt,g,m,rope", [(dict(T=2), 2, 10, False), (dict(T=2), 2, 3, True), (dict(T=3), 3, 24, False), (dict(T=2), 4, 10, True),
                                          (dict(T=2, fp8=True), 2, 10, False)], ids=str)
def test_magnitudes_of_the_other_forms(fmt, g, m, rope, spread, qs):
    """Rows whose values are put together in binary16, as stored values and queries grow and shrink."""
    pool = Pool(2, 4, 64, K=16, seed=99, spread=spread, **fmt)
    if pool.fp8:                                           # (its scales are drawn without the spread)
        pool.cent = (pool.cent.float() / spread).to(torch.bfloat16)
        spread = 1.0
    x = make(pool, 1, g, m, [250], [10], [m], seed=100, rope=rope)
    for t in ("k_new", "v_new", "tail"):
        x[t] = (x[t].float() * spread).to(torch.bfloat16)
    x["q"] = (x["q"].float() * qs).to(torch.bfloat16)
    scale = 0.1 / qs / spread
    check(pool, x, call(pool, x, softmax_scale=scale), scale=scale)


def far_pages(small, pages, n):
    """The small pool's pages at the end of a pool of `pages`, in reverse; the two sides, and the table that names them."""
    S, T, L = small.S, small.T, small.L
    e = B.alloc_cache(2, pages * L, L, small.K, small.B, T, n_smooth=S, scale_format=B.SCALE_E4M3 if small.fp8 else B.SCALE_F16)
    B.copy_pages(small.encoded(0, 2), list(range(n)), [pages - 1 - i for i in range(n)], into=e)
    half = lambda lo: B.Encoded(e.centroids[lo:lo + 1], e.ids[lo:lo + 1], e.codes[lo:lo + 1], e.scales[lo:lo + 1], L, S)      # noqa: E731
    return half(0), half(1), ints([[pages - 1 - i for i in range(n)]])


def check_far(small, sides, table, kv, g, m, rope):
    x = make(small, 1, g, m, [kv], [4], [m], seed=102, rope=rope)
    x["table"] = torch.arange(table.shape[1], dtype=torch.int32)[None]
    tail = x["tail"].cuda()
    got = B.attn_tree(x["q"].cuda(), *sides, table, ints(x["kv"]), x["k_new"].cuda(), x["v_new"].cuda(), tail_k=tail[:, :1],
                      tail_v=tail[:, 1:], tail_len=ints(x["tails"]), mask=bits_of(x["see"]).cuda(), want_lse=True,
                      k_rope=None if x["rope"] is None else x["rope"].cuda())
    check(small, x, got)


def test_codes_beyond_32_bits_in_every_form():
    L, T = 4096, 4
    pages = (1 << 32) // (L * T * 32) + 3
    small = Pool(2, 2, L, T=T, K=16, B=64, seed=101)
    *sides, table = far_pages(small, pages, 2)
    for g, m, rope in ((1, 2, False), (1, 20, False), (2, 35, False), (1, 2, True), (1, 20, True), (1, 40, True)):
        check_far(small, sides, table, L + 100, g, m, rope)


def test_tables_beyond_32_bits_in_every_form():
    L, S, K = 40, 4, 512
    pages = (1 << 32) // (S * K * D * 2) + 3
    small = Pool(2, 3, L, K=K, S=S, T=1, B=16, fp8=True, seed=103)
    *sides, table = far_pages(small, pages, 3)
    for g, m, rope in ((1, 2, False), (1, 20, False), (2, 35, False), (1, 2, True), (1, 20, True), (1, 40, True)):
        check_far(small, sides, table, 2 * L + 33, g, m, rope)
