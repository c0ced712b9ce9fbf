"""Attention over 16-bit pages against the definition in 64 bits: head sizes, types, row counts, page lengths, windows, what nobody sees."""
import math

import pytest
import torch

from paper_2602_02958_amd import binding as B
from rows_util import attention, check_attention

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F16 = torch.bfloat16, torch.float16


def gen(seed):
    return torch.Generator().manual_seed(seed)


class Case:
    """Inputs on the host; what no row of a sequence sees holds no numbers."""

    def __init__(self, kv, live, H=1, g=1, m=1, d=128, L=16, dtype=BF, causal=True, window=None, sink=0, order="head", seed=0, spread=1.0,
                 poison=True, extra=1):
        n = len(kv)
        self.kv, self.live, self.causal, self.window, self.sink = kv, [m] * n if live is None else live, causal, window, sink
        width = max(1, max(-(-x // L) for x in kv)) + extra
        P = n * width + 1
        shape = (H, P, L, d) if order == "head" else (P, L, H, d)
        self.k, self.v = (torch.randn(shape, generator=gen(seed + i)) * (spread if i == 0 else 1.0) for i in range(2))
        if order != "head":
            self.k, self.v = self.k.permute(2, 0, 1, 3), self.v.permute(2, 0, 1, 3)
        self.table = torch.randperm(P, generator=gen(seed + 2))[:n * width].view(n, width).to(torch.int32)
        if poison:
            seen = torch.zeros(P, L, dtype=torch.bool)
            for b in range(n):
                rows = max(0, min(self.live[b], m))
                lo = 0
                if window and kv[b] - rows >= window:
                    lo = kv[b] - rows - window + 1
                for t in range(kv[b]):
                    if rows and (t >= lo or t < sink):
                        seen[self.table[b, t // L], t % L] = True
            for t in (self.k, self.v):
                t[:, ~seen] = math.nan
                t[:, ~seen & (torch.arange(L) % 2 == 1)[None]] = math.inf
        self.k, self.v = self.k.to(dtype), self.v.to(dtype)
        self.q = torch.randn(n, m, H * g, d, generator=gen(seed + 3)).to(dtype).transpose(1, 2)
        self.n_new = None if live is None else torch.tensor(live, dtype=torch.int32)

    def want(self, scale=None):
        live = [max(0, min(x, self.q.shape[2])) for x in self.live]
        return attention(self.q, self.k, self.v, self.table, self.kv, live, self.causal, self.window or 0, self.sink, scale)

    def device(self):
        def there(t):
            return torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=DEV).copy_(t)
        return dict(q=there(self.q), k_pages=there(self.k), v_pages=there(self.v), page_table=self.table.to(DEV),
                    kv_len=torch.tensor(self.kv, dtype=torch.int32, device=DEV), n_new=None if self.n_new is None else self.n_new.to(DEV),
                    causal=self.causal, window=self.window, sink=self.sink)

    def check(self, scale=None):
        want, args = self.want(scale), self.device()
        for scratch in (None, torch.empty(0, dtype=torch.uint8, device=DEV)):          # divided, undivided
            out, lse = B.attn_pages(**args, want_lse=True, softmax_scale=scale, scratch=scratch)
            check_attention(out, lse, want)
        return out


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("L", [1, 16, 31, 32, 100, 256, 257, 1000])
@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
def test_head_sizes_and_page_lengths(d, L, dtype):
    Case([777, 1, 300], None, H=2, g=2, d=d, L=L, dtype=dtype, seed=1).check()


@pytest.mark.parametrize("d", [64, 128, 192, 256])
@pytest.mark.parametrize("g,m", [(1, 1), (7, 1), (16, 1), (17, 1), (1, 33), (4, 5), (8, 8), (3, 40)])
def test_row_counts(g, m, d):
    """Blocks of 16 and 32 rows, several of them, full or not; heads' rows side by side."""
    Case([613, 40, 5], [m, max(1, m // 2), m], H=2, g=g, m=m, d=d, L=48, seed=2).check()
    Case([130, 600], [m, 1], H=1, g=g, m=m, d=d, L=320, dtype=F16, causal=False, order="token", seed=3).check()


@pytest.mark.parametrize("d,dtype", [(64, BF), (96, F16), (128, BF), (192, F16), (256, BF)])
def test_many_rows(d, dtype):
    """Rows of wavefronts' own, blocks of them that are not full, divided and not; pages of both kinds."""
    Case([700, 350, 0, 33], [20, 20, 20, 7], H=2, g=16, m=20, d=d, L=24, dtype=dtype, seed=44).check()
    Case([1500], [65], H=1, g=1, m=65, d=d, L=300, dtype=dtype, order="token", seed=45).check()
    Case([1500, 2], [100, 3], H=1, g=3, m=100, d=d, L=32, dtype=dtype, window=300, sink=50, seed=46).check()


@pytest.mark.parametrize("kv", [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1023, 1025, 2049])
@pytest.mark.parametrize("L", [16, 64, 300])
def test_lengths(kv, L):
    Case([kv, max(0, kv - 1)], None, H=1, g=3, L=L, seed=4).check()


@pytest.mark.parametrize("L", [8, 32, 50, 256, 330])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (5, 3), (31, 0), (32, 32), (33, 31), (64, 40), (100, 200), (300, 7), (1 << 33, 5), (2000, 0)])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(window, sink, L, causal):
    Case([700, 33, 1, 350, 64], [4, 4, 4, 1, 0], H=2, g=2, m=4, L=L, window=window, sink=sink, causal=causal, d=64, seed=5).check()


@pytest.mark.parametrize("window,sink", [(40, 10), (10, 500)])
def test_windows_of_many_rows(window, sink):
    Case([400, 90], [70, 70], H=1, g=1, m=70, L=40, window=window, sink=sink, seed=6).check()
    Case([400, 20], [70, 33], H=1, g=2, m=70, L=288, window=window, sink=sink, causal=False, seed=7).check()


def test_rows_before_the_sequence_and_counts_beyond_their_range():
    """More new tokens than the cache holds: rows at negative places see nothing (causal); counts and lengths are clamped."""
    Case([3, 40, 0, 10], [8, 99, 8, -2], H=1, g=2, m=8, L=16, seed=8).check()
    Case([3, 40, 0, 10], [8, 99, 8, -2], H=1, g=2, m=8, L=16, causal=False, seed=9).check()
    c = Case([64, 64], None, L=16, seed=10, extra=0, poison=False)
    args = c.device()
    args["kv_len"] = torch.tensor([1 << 30, -7], dtype=torch.int32, device=DEV)
    c.kv = [64, 0]
    out, lse = B.attn_pages(**args, want_lse=True)
    check_attention(out, lse, c.want())


def test_pages_outside_the_pool_read_the_nearest():
    c = Case([100, 100], None, L=32, seed=11, poison=False)
    c.table[0, 1], c.table[1, 0] = -5, 1 << 30
    c.check()


def test_pages_behind_the_sequence_and_before_its_window_are_not_looked_at():
    c = Case([500, 70], [2, 2], m=2, L=16, window=60, sink=20, seed=12)
    c.check()
    args = c.device()
    want = B.attn_pages(**args)
    for b, kv in enumerate(c.kv):
        lo = kv - 2 - 60 + 1
        for p in range(c.table.shape[1]):
            if p * 16 >= kv or (p * 16 >= 20 and (p + 1) * 16 <= lo):
                args["page_table"][b, p] = -(1 << 31)
    assert torch.equal(B.attn_pages(**args), want)


@pytest.mark.parametrize("dtype", [BF, F16])
def test_scores_of_every_size(dtype):
    """Equal keys, sharp rows, scores beyond 2^24, rows of one token that outweighs the others."""
    c = Case([300, 700], None, H=2, g=2, L=16, dtype=dtype, seed=13, spread=30.0)
    c.check()
    c = Case([600], None, H=1, g=1, L=16, dtype=dtype, seed=14, poison=False)
    c.k[:] = 0.5
    c.check()
    c = Case([400], None, H=1, g=2, L=16, dtype=dtype, seed=15, poison=False)
    c.q.mul_(100), c.k.mul_(100)
    c.check()
    # exact scores that leave fp32's whole numbers: q and k have one channel, tokens 37 and 38 share the largest
    c = Case([200], None, H=1, g=1, L=32, dtype=dtype, seed=16, poison=False)
    c.q.zero_(), c.k.zero_()
    c.q[..., 3] = 2.0 ** 14
    flat = c.table[0].long()
    k = c.k[0, flat].flatten(0, 1)
    k[:, 3] = -(2.0 ** 14)
    k[37, 3] = k[38, 3] = 2.0 ** 14
    k[39, 3] = 2.0 ** 14 * (1 - 2.0 ** -5)
    c.k[0, flat] = k.view(flat.shape[0], 32, 128)
    out, lse = B.attn_pages(**c.device(), want_lse=True, softmax_scale=1.0)
    v = c.v[0, flat].flatten(0, 1).double()
    want = (v[37] + v[38]) / 2
    assert ((out[0, 0, 0].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20).all()
    assert abs(float(lse) - 2.0 ** 28) <= 2.0 ** 28 * 2.0 ** -22


def test_scales():
    for scale in (1e-3, 0.7):
        Case([90, 513], None, H=1, g=4, L=64, seed=17).check(scale)


def test_small_numbers_keep_their_bits():
    """Subnormal values of binary16, and products that far below 1."""
    c = Case([300, 40], None, H=1, g=2, L=16, dtype=F16, seed=40, poison=False)
    c.v.mul_(2.0 ** -16)
    c.k.mul_(2.0 ** -14)
    c.check()
    c.check(scale=2.0 ** 12)
    c = Case([300, 40], None, H=1, g=2, L=16, dtype=BF, seed=41, poison=False)
    c.v.mul_(2.0 ** -100)
    c.q.mul_(2.0 ** -60), c.k.mul_(2.0 ** -60)
    c.check()


def test_large_scales_and_small_ones():
    c = Case([200, 30], None, H=1, g=2, L=16, seed=42)
    c.check(scale=1e-44)
    c.check(scale=1e-38)
    # products of at most 1 / 128, of which one is a power of two above the others
    c = Case([200], None, H=1, g=1, L=32, seed=43, poison=False)
    c.q.zero_(), c.k.zero_()
    c.q[..., 0] = 2.0 ** -10
    flat = c.table[0].long()
    k = c.k[0, flat].flatten(0, 1)
    k[:, 0] = 2.0 ** -11
    k[77, 0] = 2.0 ** -10
    c.k[0, flat] = k.view(flat.shape[0], 32, 128)
    for scratch in (None, torch.empty(0, dtype=torch.uint8, device=DEV)):
        out = B.attn_pages(**c.device(), softmax_scale=2.0 ** 100, scratch=scratch)
        assert torch.equal(out[0, 0, 0].cpu(), c.v[0, flat].flatten(0, 1)[77])


def test_one_sequence_many_parts_and_many_sequences():
    Case([5000], None, H=1, g=1, L=48, seed=18).check()
    Case([4000, 3, 2500], None, H=1, g=2, L=512, d=64, seed=19).check()
    kv = [(i * 37) % 90 for i in range(70)]
    Case(kv, None, H=1, g=2, d=64, L=16, seed=20).check()
    kv = [(i * 37) % 90 for i in range(300)]              # (more than are divided)
    kv[7] = 900
    Case(kv, None, H=1, g=1, d=64, L=16, seed=21).check()
    # many workgroups: only sequences much longer than the others are divided
    Case([5000 if i == 13 else 40 + i for i in range(70)], None, H=8, g=1, d=64, L=32, seed=36).check()
    Case([2600 if i in (0, 63) else 0 for i in range(64)], None, H=16, g=2, d=64, L=32, seed=37).check()
    Case([900] * 40, None, H=8, g=1, d=64, L=64, seed=38).check()
    kv = [600 if i % 50 == 0 else i % 4 for i in range(200)]
    Case(kv, None, H=1, g=1, d=64, L=64, seed=22).check()


def test_scratch_is_lent_and_equal_calls_give_equal_bits():
    c = Case([3000, 700], None, H=2, g=2, L=64, seed=23)
    args = c.device()
    scratch = B.attn_pages_scratch(args["k_pages"], 2, 2, 1, c.table.shape[1])
    assert scratch.numel() > 0
    first = B.attn_pages(**args, scratch=scratch)
    scratch.fill_(255)
    assert torch.equal(B.attn_pages(**args, scratch=scratch), first)
    assert torch.equal(B.attn_pages(**args), first)


def test_out_may_be_q_and_has_strides_of_its_own():
    c = Case([300, 20], [3, 2], H=2, g=2, m=3, L=16, seed=24)
    args = c.device()
    want = B.attn_pages(**args)
    room = torch.full((2, 4, 3, 136), 7.0, dtype=BF, device=DEV)
    out = room[..., :128]
    assert B.attn_pages(**args, out=out) is out
    assert torch.equal(out, want) and (room[..., 128:] == 7).all()
    args["q"] = args["q"].contiguous()
    assert torch.equal(B.attn_pages(**args, out=args["q"]), want)


def test_no_sequences_no_rows_no_pages():
    c = Case([20], None, L=16, seed=25)
    a = c.device()
    assert B.attn_pages(a["q"][:0], a["k_pages"], a["v_pages"], a["page_table"][:0], a["kv_len"][:0]).shape == (0, 1, 1, 128)
    assert B.attn_pages(a["q"][:, :, :0], a["k_pages"], a["v_pages"], a["page_table"], a["kv_len"]).shape == (1, 1, 0, 128)
    out, lse = B.attn_pages(a["q"], a["k_pages"], a["v_pages"], a["page_table"][:, :0].contiguous(), a["kv_len"], want_lse=True)
    assert not out.any() and (lse == -math.inf).all()


def test_a_pool_beyond_4_gib():
    """Pages and tokens whose rows lie beyond 2^32 bytes."""
    H, P, L, d = 2, 9, 1 << 20, 128
    kp, vp = (torch.empty(H, P, L, d, dtype=BF, device=DEV).fill_(math.nan) for _ in range(2))
    q = torch.randn(1, H, 1, d, generator=gen(30)).to(BF)
    k, v = (torch.randn(H, 50, d, generator=gen(i)).to(BF) for i in (31, 32))
    kp[:, 8, L - 50:], vp[:, 8, L - 50:] = k.to(DEV), v.to(DEV)
    out, lse = B.attn_pages(q.to(DEV), kp, vp, torch.tensor([[8]], dtype=torch.int32, device=DEV), torch.tensor([L], dtype=torch.int32, device=DEV),
                            window=50, want_lse=True)
    small = attention(q, k[:, None], v[:, None], torch.zeros(1, 1, dtype=torch.int32), [50], [1])
    check_attention(out, lse, small)
    # a token's stride of 2^20 elements
    wide = torch.empty(1, 1, 40, 1 << 20, dtype=BF, device=DEV)
    kp, vp = wide[..., :128], wide[..., 512:640]
    kp.copy_(k[:1, None, :40].to(DEV)), vp.copy_(v[:1, None, :40].to(DEV))
    out, lse = B.attn_pages(q[:, :1].to(DEV), kp, vp, torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.tensor([40], dtype=torch.int32, device=DEV),
                            want_lse=True)
    check_attention(out, lse, attention(q[:, :1], k[:1, None, :40], v[:1, None, :40], torch.zeros(1, 1, dtype=torch.int32), [40], [1]))


def test_two_graphs_that_share_their_scratch():
    c = Case([3000, 100], None, H=1, g=2, L=64, seed=33)
    args = c.device()
    scratch = B.attn_pages_scratch(args["k_pages"], 2, 2, 1, c.table.shape[1])
    q2 = torch.randn(c.q.shape, generator=gen(34)).to(BF).to(DEV)
    outs = [torch.empty(2, 2, 1, 128, dtype=BF, device=DEV) for _ in range(2)]
    B.attn_pages(**args, scratch=scratch, out=outs[0])
    torch.cuda.synchronize()
    graphs = []
    for q, out in ((args["q"], outs[0]), (q2, outs[1])):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.attn_pages(**{**args, "q": q}, scratch=scratch, out=out)
        graphs.append(g)
    for i in range(4):
        args["kv_len"].copy_(torch.tensor([3000 - 700 * i, 100 + i], dtype=torch.int32))
        for out in outs:
            out.zero_()
        for g in graphs:
            g.replay()
        for q, out in ((args["q"], outs[0]), (q2, outs[1])):
            assert torch.equal(out, B.attn_pages(**{**args, "q": q}))
        torch.cuda.synchronize()


def test_on_another_stream():
    c = Case([2000], None, H=2, g=2, L=64, seed=35)
    args = c.device()
    want = B.attn_pages(**args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = B.attn_pages(**args)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
