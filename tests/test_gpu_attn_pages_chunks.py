"""Attention over 16-bit pages of a chunk's or a prompt's queries: thousands of rows of a KV head, hundreds of blocks of them, against the
definition in 64 bits (on the device, where so many rows are quick)."""
import math

import pytest
import torch

from paper_2602_02958_amd import binding as B
from rows_util import HALF_STEP, TINY, turned, within
from test_gpu_pages_rollout import Program

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F16 = torch.bfloat16, torch.float16


def rows_on_device(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def check(q, kp, vp, table, kv_len, live, out, lse, causal=True, window=0, sink=0, block=512):
    """out and lse [B, Hq, N, ..] against attention in 64 bits, `block` rows at a time; the bounds are those of rows_util.attention."""
    n, hq, m, d = q.shape
    H, _, L, _ = kp.shape
    scale = 1 / math.sqrt(d)
    for b in range(n):
        kv, rows = kv_len[b], live[b]
        assert not out[b, :, rows:].any() and (lse[b, :, rows:] == -math.inf).all()
        pages, t = table[b, :-(-kv // L)].long(), torch.arange(kv, device=DEV)
        sums = (kv / 16 + 64) * 2.0 ** -23
        for h in range(hq):
            K, V = (p[h * H // hq, pages].flatten(0, 1)[:kv].double() for p in (kp, vp))
            top = V.abs().amax()
            for i in range(0, rows, block):
                at = torch.arange(i, min(i + block, rows), device=DEV)
                place = (kv - rows + at)[:, None]
                see = t <= place if causal else torch.ones(len(at), kv, dtype=torch.bool, device=DEV)
                if window:
                    see = see & ((t > place - window) | (t < sink))
                x = q[b, h, at].double()
                s = (scale * (x @ K.T)).masked_fill(~see, -math.inf)
                e = scale * (x.abs() @ K.abs().T).masked_fill(~see, 0).amax(1) * (d + 32) * 2.0 ** -23
                z = torch.logsumexp(s, 1)
                w = torch.exp(s - z[:, None])
                o = w @ V
                tol = HALF_STEP[q.dtype] * o.abs() + (torch.expm1(2 * e)[:, None] + 2.0 ** -15 + sums) * (w @ V.abs()) + TINY[q.dtype]
                if q.dtype is F16:
                    tol = tol + 2.0 ** -19 * top         # 32 times 2^-24 of the largest weight of a tile, of all tiles
                far = ((out[b, h, at].double() - o).abs() - tol).max()
                assert far <= 0, f"sequence {b} head {h} rows from {i}: off by {float(far):.3e} more than allowed"
                assert ((lse[b, h, at].double() - z).abs() <= e + 2.0 ** -20 * (1 + z.abs()) + sums).all(), (b, h, i)


@pytest.mark.parametrize("kv,live,H,g,m,d,L,dtype,causal,window,sink", [
    ([9360], None, 2, 1, 4680, 128, 4680, BF, True, 0, 0),                         # a chunk behind another
    ([2048, 300], [1024, 300], 1, 4, 1024, 128, 64, BF, True, 0, 0),               # prompts: the second from its first token on
    ([6000], None, 1, 1, 4680, 64, 1000, F16, False, 0, 0),
    ([4000, 77, 2500], [2000, 50, 2000], 2, 1, 2000, 64, 100, F16, True, 64, 5),   # a window of few tokens, many rows
    ([3000, 1500], [1111, 1500], 1, 3, 1500, 96, 48, BF, True, 700, 40),
    ([2000], None, 1, 2, 1000, 192, 64, F16, True, 0, 0), ([2000, 900], None, 1, 2, 777, 256, 32, BF, True, 130, 3),
    ([5000] * 3, [10, 600, 1], 8, 1, 600, 64, 16, BF, True, 0, 0),
])
def test_chunks(kv, live, H, g, m, d, L, dtype, causal, window, sink):
    n, width = len(kv), -(-max(kv) // L)
    live = [m] * n if live is None else live
    kp, vp = (rows_on_device((H, n * width, L, d), dtype, s) for s in (1, 2))
    q = rows_on_device((n, m, H * g, d), dtype, 3).transpose(1, 2)
    table = torch.randperm(n * width, generator=torch.Generator().manual_seed(4)).view(n, width).to(torch.int32).to(DEV)
    out, lse = B.attn_pages(q, kp, vp, table, torch.tensor(kv, dtype=torch.int32, device=DEV), torch.tensor(live, dtype=torch.int32, device=DEV), causal=causal,
                            window=window or None, sink=sink, want_lse=True)
    check(q, kp, vp, table, kv, live, out, lse, causal, window, sink)


def test_as_many_rows_as_a_call_takes():
    """2^20 query rows of a KV head, 32768 blocks; of 2 heads."""
    d, L = 64, 16
    kp, vp = (rows_on_device((2, 3, L, d), BF, s) for s in (5, 6))
    q = rows_on_device((1, 2 * 1024, 1024, d), BF, 7)
    table, kv = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV), torch.tensor([35], dtype=torch.int32, device=DEV)
    out, lse = B.attn_pages(q, kp, vp, table, kv, causal=False, want_lse=True)
    check(q, kp, vp, table, [35], [1024], out, lse, causal=False, block=1024)


@pytest.mark.parametrize("window,sink", [(None, 0), (1560, 52)])
def test_a_step_of_chunks(window, sink):
    """table, turned queries, appended keys and values, attention: a chunk of 4680 tokens, another, and one token."""
    p = Program(1, 2, 1, 128, 4680, 3, 64, False, BF, window, sink)
    held = 0
    for i, n in enumerate((4680, 4680, 1)):
        q, k, v = (rows_on_device((1, n, 2, 128), BF, 10 * i + s).transpose(1, 2) for s in range(3))
        turned_q = B.rope(q, p.rotary, first=p.len)
        out, lse = p.step(q, k, v)
        assert p.len.tolist() == [held + n]
        page = int(p.table[0, held // 4680])
        at = slice(held % 4680, held % 4680 + n)
        assert torch.equal(p.v[:, page, at], v[0])
        want, tol = turned(k[0].cpu(), p.rotary[held:held + n].cpu())
        within(p.k[:, page, at], want, tol)
        held += n
        check(turned_q, p.k, p.v, p.table, [held], [n], out, lse, True, window or 0, sink)
