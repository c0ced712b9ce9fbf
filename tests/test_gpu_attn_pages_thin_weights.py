"""Many tokens of weights that are far below their row's largest, over pages of 16 bits: what they add up to is a part of the sum, in binary16
too, whose numbers end at 2^-24."""
import math

import pytest
import torch

from paper_2602_02958_amd import binding as B
from rows_util import HALF_STEP, TINY

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F16 = torch.bfloat16, torch.float16
HEAVY = {"first": lambda n: [0, 33, 70, 100], "one": lambda n: [5], "scattered": lambda n: list(range(3, n, n // 40)), "last": lambda n: [n - 1]}


def exact(score, v, tile=32):
    """One row of scores (exact numbers) over values [N, d] in 64 bits -> out, lse, the bounds of both.

    A score is exact, its product with the scale and log2 e off by 2^-22 of it, and so a weight by e = 2^-22 |score - largest| and 2^-21.  It
    enters as two numbers of the type: off by 2^-16 (bf16) or 2^-22 (binary16) of itself, in binary16 otherwise by 2^-24 of the largest of its
    tile's, or by all of itself if that is less.  A product passes 2 (N / 32) + 64 fp32 sums, a weight as many."""
    n = score.shape[0]
    z = torch.logsumexp(score, 0)
    w = torch.exp(score - z)
    e = (score - score.max()).abs() * 2.0 ** -22
    top = torch.nn.functional.pad(w, (0, -n % tile)).view(-1, tile).amax(1).repeat_interleave(tile)[:n]
    sums = (n / 16 + 64) * 2.0 ** -23
    out, mag = w @ v, w @ v.abs()
    off = (w * (2 * torch.expm1(e) + 2.0 ** -15)) @ v.abs() + sums * mag + float((w * torch.expm1(e)).sum()) * out.abs()
    thin = torch.minimum(w, 2.0 ** -24 * top) @ v.abs()
    return out, z, off, thin, 2.0 ** -20 * (1 + z.abs()) + sums


def rows_of(case, n, d, dtype, seed):
    """Keys [n, d] of one channel, whose scores are far below the heavy tokens', and values, large where weights are small."""
    g = torch.Generator().manual_seed(seed)
    score = -torch.full((n,), 23.0, dtype=torch.float64)
    if case[1]:                                              # spread over 2^-4 .. 2^-52 of the largest, tile by tile
        score = -torch.randint(3, 36, (-(-n // 32),), generator=g).double().repeat_interleave(32)[:n]
    v = torch.where(score[:, None] < -15, 30000.0, 1.0) * (1 + torch.rand(n, d, generator=g, dtype=torch.float64))
    heavy = HEAVY[case[0]](n)
    score[heavy] = 0.0
    v[heavy] *= 2.0 ** -20
    k = torch.zeros(n, d, dtype=dtype)
    k[:, 0] = score.to(dtype)
    assert torch.equal(k[:, 0].double(), score)
    return k, v.to(dtype), score


@pytest.mark.parametrize("heavy", HEAVY)
@pytest.mark.parametrize("spread", [False, True])
@pytest.mark.parametrize("d,dtype,g,m,L", [(128, F16, 1, 1, 64), (64, F16, 3, 7, 100), (96, F16, 17, 1, 48), (192, F16, 2, 3, 4096), (256, F16, 8, 3, 32),
                                           (128, BF, 1, 2, 64)])
def test_thin_weights(d, dtype, g, m, L, spread, heavy):
    n = 60000
    k, v, score = rows_of((heavy, spread), n, d, dtype, 7)
    pages = -(-n // L)
    kp, vp = (torch.zeros(1, pages, L, d, dtype=dtype) for _ in range(2))
    for pool, x in ((kp, k), (vp, v)):
        pool.view(pages * L, d)[:n] = x
    q = torch.zeros(1, g, m, d, dtype=dtype)
    q[..., 0] = 1.0
    args = dict(page_table=torch.arange(pages, dtype=torch.int32, device=DEV)[None], kv_len=torch.tensor([n], dtype=torch.int32, device=DEV),
                softmax_scale=1.0, causal=False, want_lse=True)
    out, z, off, thin, ltol = exact(score, v.double())
    tol = HALF_STEP[dtype] * out.abs() * (1 + 2.0 ** -10) + off + TINY[dtype] + (thin if dtype is F16 else 0.0)
    assert (tol <= 0.1 * out.abs()).all()                    # (what is lost below 2^-24 of the whole is more than that)
    for scratch in (None, torch.empty(0, dtype=torch.uint8, device=DEV)):
        got, lse = B.attn_pages(q.to(DEV), kp.to(DEV), vp.to(DEV), **args, scratch=scratch)
        far = (got.cpu().double() - out).abs() - tol
        assert torch.isfinite(got.float()).all() and (far <= 0).all(), f"off by {float(far.max()):.3e} more than allowed of {float(out.abs().max()):.3e}"
        assert ((lse.cpu().double() - z).abs() <= ltol).all()


def test_rows_of_a_block_that_are_lifted_apart():
    """Rows of one block whose weights lie far apart, beside rows that see nothing of a tile: each as alone."""
    n, d, m, L = 2000, 64, 32, 32
    g = torch.Generator().manual_seed(3)
    kp, vp = (torch.randn(1, 63, L, d, generator=g).to(F16) for _ in range(2))
    q = torch.randn(1, 1, m, d, generator=g).to(F16) * torch.logspace(-3, 1.5, m)[None, None, :, None].to(F16)
    table, lens = torch.arange(63, dtype=torch.int32, device=DEV)[None], torch.tensor([n], dtype=torch.int32, device=DEV)
    none = torch.empty(0, dtype=torch.uint8, device=DEV)
    for window in (None, 300):
        whole, lse = B.attn_pages(q.to(DEV), kp.to(DEV), vp.to(DEV), table, lens, causal=False, window=window, want_lse=True, scratch=none)
        K, V = (t.view(-1, d)[:n].double() for t in (kp, vp))
        for i in range(m):
            see = torch.arange(n) > (n - m + i - window if window else -1)
            s = (K @ q[0, 0, i].double()) / math.sqrt(d)
            s = s.masked_fill(~see, -math.inf)
            z = torch.logsumexp(s, 0)
            w = torch.exp(s - z)
            e = float((K.abs() @ q[0, 0, i].double().abs()).max()) / math.sqrt(d) * (d + 32) * 2.0 ** -23
            sums = (n / 16 + 64) * 2.0 ** -23
            tol = HALF_STEP[F16] * (w @ V).abs() + (math.expm1(2 * e) + 2.0 ** -15 + sums) * (w @ V.abs()) + 2.0 ** -19 * V.abs().max() + TINY[F16]
            assert ((whole[0, 0, i].cpu().double() - w @ V).abs() <= tol).all(), i
            assert abs(float(lse[0, 0, i]) - float(z)) <= e + 2.0 ** -20 * (1 + abs(float(z))) + sums, i
