"""New tokens on their way into 16-bit pages: every row of the pool against the definition, those that nobody writes bit for bit."""
import pytest
import torch

from paper_2602_02958_amd import binding as B
from rows_util import turned, within

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def gen(seed):
    return torch.Generator().manual_seed(seed)


def pool_of(heads, pages, L, d, dtype, order="head", seed=0):
    """(K, V) pages [H, P, L, d] on the host, unit-major or a token's heads side by side."""
    shape = (heads, pages, L, d) if order == "head" else (pages, L, heads, d)
    both = [torch.randn(shape, generator=gen(seed + i)).to(dtype) for i in range(2)]
    return both if order == "head" else [t.permute(2, 0, 1, 3) for t in both]


def on_device(t):
    """The same view on the device."""
    out = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=DEV)
    return out.copy_(t)


def check(pool, k, v, table, kv, live, got_k, got_v, new_len, rot=None, half=False, positions=None):
    """pool: (K, V) before, k, v [B, H, N, d]."""
    H, P, L, d = pool[0].shape
    want = [t.clone().double() for t in pool]
    tol = torch.zeros_like(want[0])
    cap = table.shape[1] * L
    lens = []
    for b in range(k.shape[0]):
        at = min(max(int(kv[b]), 0), cap)
        n = min(max(int(live[b]), 0), k.shape[2])
        lens.append(min(at + n, cap))
        for i in range(min(n, cap - at)):
            page = int(table[b, (at + i) // L])
            if not 0 <= page < P:
                continue
            row = k[b, :, i]
            val, t = row.double(), torch.zeros_like(row.double())
            if rot is not None:
                place = at + i if positions is None else int(positions[b, i])
                val, t = turned(row, rot[min(max(place, 0), rot.shape[0] - 1)][None], half)
            want[0][:, page, (at + i) % L], tol[:, page, (at + i) % L] = val, t
            want[1][:, page, (at + i) % L] = v[b, :, i].double()
    within(got_k, want[0], tol)
    assert torch.equal(got_v.cpu().double(), want[1])
    assert new_len.tolist() == lens


def tables(seqs, width, pages, seed):
    """Pages that no two entries share."""
    assert seqs * width <= pages
    return torch.randperm(pages, generator=gen(seed))[:seqs * width].view(seqs, width).to(torch.int32)


def rotary(n, pairs, dtype, seed):
    ang = torch.rand(n, pairs, generator=gen(seed), dtype=torch.float64) * 50
    return torch.stack([ang.cos(), ang.sin()], -1).to(dtype)


CASES = [  # B, H, N, d, L, kv, live
    (1, 1, 1, 128, 1, [3], None), (3, 2, 1, 128, 16, [0, 15, 16], None), (2, 3, 70, 64, 7, [5, 0], [70, 13]), (4, 2, 9, 96, 32, [0, 31, 95, 96], [9, 0, 9, 4]),
    (1, 12, 300, 128, 100, [250], None), (2, 1, 33, 256, 24, [1, 23], [33, 1]), (5, 4, 6, 40, 5, [9, 8, 7, 6, 5], [-3, 0, 6, 99, 2]),
]


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("turn", [None, ("all", False), ("all", True), ("part", False), ("part", True), ("odd", True), ("odd", False)])
@pytest.mark.parametrize("case", CASES)
def test_rows_go_where_they_belong(case, turn, dtype, order):
    n, H, m, d, L, kv, live = case
    width = max(-(-(a + m) // L) for a in kv) + 1
    pool = pool_of(H, n * width + 2, L, d, dtype, order, 1)
    k, v = (torch.randn(n, m, H, d, generator=gen(i)).to(dtype).transpose(1, 2) for i in (3, 4))
    table, lens = tables(n, width, n * width + 2, 5), torch.tensor(kv, dtype=torch.int32)
    pairs = {"all": d // 2, "part": d // 4, "odd": d // 2 - 3}[turn[0]] if turn else 0
    half = bool(turn and turn[1])
    rot = rotary(width * L, pairs, F32 if dtype is F16 else F16, 6) if turn else None
    kp, vp = (on_device(t) for t in pool)
    kd, vd = (on_device(t) for t in (k, v))
    n_new = None if live is None else torch.tensor(live, dtype=torch.int32)
    got = B.append_pages(kd, vd, kp, vp, table.to(DEV), lens.to(DEV), None if n_new is None else n_new.to(DEV),
                         None if rot is None else rot.to(DEV), half=half)
    check(pool, k, v, table, kv, [m] * n if live is None else live, kp, vp, got, rot, half)
    assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)


def test_given_positions_and_places_beyond_the_rotary_table():
    pool = pool_of(2, 6, 8, 128, BF, seed=10)
    k, v = (torch.randn(2, 2, 5, 128, generator=gen(i)).to(BF) for i in (11, 12))
    table, kv, rot = tables(2, 3, 6, 13), torch.tensor([2, 9], dtype=torch.int32), rotary(10, 64, F16, 14)
    pos = torch.tensor([[0, 3, 3, -7, 99], [1, 2, 9, 10, 5]], dtype=torch.int32)
    for p in (pos, None):
        kp, vp = (on_device(t) for t in pool)
        got = B.append_pages(k.to(DEV), v.to(DEV), kp, vp, table.to(DEV), kv.to(DEV), k_rope=rot.to(DEV), positions=None if p is None else p.to(DEV))
        check(pool, k, v, table, kv, [5, 5], kp, vp, got, rot, positions=p)


def test_tokens_beyond_the_table_and_pages_outside_the_pool_are_left_out():
    pool = pool_of(2, 5, 4, 64, BF, seed=20)
    k, v = (torch.randn(4, 2, 9, 64, generator=gen(i)).to(BF) for i in (21, 22))
    table = torch.tensor([[0, -1, 1], [2, 5, 3], [4, 1 << 30, -(1 << 31)], [-1, -1, -1]], dtype=torch.int32)
    kv = torch.tensor([0, 7, -5, 1 << 30], dtype=torch.int32)
    kp, vp = (on_device(t) for t in pool)
    got = B.append_pages(k.to(DEV), v.to(DEV), kp, vp, table.to(DEV), kv.to(DEV))
    check(pool, k, v, table, kv, [9] * 4, kp, vp, got)
    assert got.tolist() == [9, 12, 9, 12]


def test_lengths_in_place_and_without_tokens():
    pool = pool_of(1, 8, 4, 64, BF, seed=30)
    k, v = (torch.randn(300, 1, 3, 64, generator=gen(i)).to(BF).to(DEV) for i in (31, 32))
    table = torch.full((300, 4), -1, dtype=torch.int32, device=DEV)
    kv = torch.arange(300, dtype=torch.int32, device=DEV) % 20
    live = torch.arange(300, dtype=torch.int32, device=DEV) % 5 - 1
    want = (kv.clamp(0, 16) + live.clamp(0, 3)).clamp(max=16)
    kp, vp = (on_device(t) for t in pool)
    assert torch.equal(B.append_pages(k, v, kp, vp, table, kv, live), want)
    both = kv.clone()
    assert B.append_pages(k, v, kp, vp, table, both, live, out_len=both) is both and torch.equal(both, want)
    there = live.clone()                                     # (over the counts)
    B.append_pages(k, v, kp, vp, table, kv, there, out_len=there)
    assert torch.equal(there, want)
    none = k[:, :, :0]
    assert torch.equal(B.append_pages(none, none, kp, vp, table, kv), kv.clamp(0, 16))
    assert B.append_pages(k[:0], v[:0], kp, vp, table[:0], kv[:0]).shape == (0,)
    assert torch.equal(B.append_pages(k, v, kp, vp, table[:, :0].contiguous(), kv), torch.zeros_like(kv))
    assert torch.equal(kp.cpu(), pool[0]) and torch.equal(vp.cpu(), pool[1])


def test_values_that_are_no_numbers_are_copied():
    pool = pool_of(1, 2, 4, 64, BF, seed=40)
    k, v = (torch.full((1, 1, 2, 64), float("nan"), dtype=BF) for _ in range(2))
    kp, vp = (on_device(t) for t in pool)
    B.append_pages(k.to(DEV), v.to(DEV), kp, vp, torch.tensor([[1]], dtype=torch.int32, device=DEV), torch.tensor([1], dtype=torch.int32, device=DEV))
    assert kp[0, 1, 1:3].isnan().all() and vp[0, 1, 1:3].isnan().all()
    assert torch.equal(kp[0, 0].cpu(), pool[0][0, 0]) and torch.equal(kp[0, 1, 3:].cpu(), pool[0][0, 1, 3:])


def test_a_pool_beyond_4_gib():
    """Pages whose rows lie beyond 2^32 bytes, and token strides beyond 2^16."""
    H, P, L, d = 2, 9, 1 << 20, 128
    kp, vp = (torch.zeros(H, P, L, d, dtype=BF, device=DEV) for _ in range(2))
    k, v = (torch.randn(1, H, 3, d, generator=gen(i)).to(BF) for i in (50, 51))
    table = torch.tensor([[8]], dtype=torch.int32, device=DEV)
    got = B.append_pages(k.to(DEV), v.to(DEV), kp, vp, table, torch.tensor([L - 2], dtype=torch.int32, device=DEV))
    assert got.tolist() == [L]
    assert torch.equal(kp[:, 8, L - 2:].cpu(), k[0, :, :2]) and torch.equal(vp[:, 8, L - 2:].cpu(), v[0, :, :2])
    assert not kp[:, :8].any() and not kp[:, 8, :L - 2].any()


def test_in_a_graph_steps_follow_each_other():
    pool = pool_of(2, 8, 4, 64, BF, seed=60)
    kp, vp = (on_device(t) for t in pool)
    k, v = (torch.randn(2, 2, 1, 64, generator=gen(i)).to(BF).to(DEV) for i in (61, 62))
    table = tables(2, 4, 8, 63).to(DEV)
    rot = rotary(16, 32, F16, 64).to(DEV)
    kv = torch.zeros(2, dtype=torch.int32, device=DEV)
    B.append_pages(k, v, kp.clone(), vp.clone(), table, kv, k_rope=rot, out_len=kv.clone())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.append_pages(k, v, kp, vp, table, kv, k_rope=rot, out_len=kv)
    want_k, want_v, lens = kp.clone(), vp.clone(), kv.clone()
    for i in range(9):
        k.copy_(torch.randn(2, 2, 1, 64, generator=gen(70 + i)))
        v.copy_(torch.randn(2, 2, 1, 64, generator=gen(90 + i)))
        B.append_pages(k, v, want_k, want_v, table, lens, k_rope=rot, out_len=lens)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(kp, want_k) and torch.equal(vp, want_v) and torch.equal(kv, lens)
    assert kv.tolist() == [9, 9]
