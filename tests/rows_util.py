"""What the tests of the rotary operators and of the caches of 16-bit pages share: the operators in 64 bits on the host, written from
their definitions, and bounds on what a kernel may be off."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24, torch.float64: 2.0 ** -53}     # of a rounding, relative
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149, torch.float64: 0.0}        # and where the type's steps end


def turned(x, cs, half=False, backward=False):
    """Rows x [.., d] by (cos, sin) cs [.., P, 2] in 64 bits, and the bound of a turned row that is rounded to x's type: an fp32 product, an fp32
    fma (2^-24 of each term and of their sum), one rounding to the type."""
    p, d = cs.shape[-2], x.double()
    c, s = cs.double().unbind(-1)
    if backward:
        s = -s
    lo, hi = (slice(0, p), slice(p, 2 * p)) if half else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
    y, mag = d.clone(), torch.zeros_like(d)
    y[..., lo], y[..., hi] = c * d[..., lo] - s * d[..., hi], s * d[..., lo] + c * d[..., hi]
    mag[..., lo] = (c * d[..., lo]).abs() + (s * d[..., hi]).abs()
    mag[..., hi] = (s * d[..., lo]).abs() + (c * d[..., hi]).abs()
    tol = HALF_STEP[x.dtype] * y.abs() * (1 + 2.0 ** -10) + 2.0 ** -23 * mag + TINY[x.dtype]
    tol[mag == 0] = 0.0                                    # what is not turned is kept bit for bit
    tol[..., 2 * p:] = 0.0
    return y, tol


def within(got, want, tol):
    off = (got.detach().cpu().double() - want).abs() - tol
    assert torch.isfinite(got.detach().float()).all()
    assert (off <= 0).all(), f"off by {float(off.max()):.3e} more than allowed at {int(off.argmax())}"


def sees(kv, live, causal, window, sink):
    """[live, kv] bool: what row i of a sequence sees."""
    t, place = torch.arange(kv)[None], (kv - live + torch.arange(live))[:, None]
    see = t <= place if causal else torch.ones(live, kv, dtype=torch.bool)
    if window:
        see = see & ((t > place - window) | (t < sink))
    return see


def tokens_of(pool, table, kv):
    """[H, kv, d] of a sequence, from pages [H, P, L, d] on the host."""
    L = pool.shape[2]
    n = -(-kv // L)
    pages = table[:n].long().clamp(0, pool.shape[1] - 1)
    return pool[:, pages].flatten(1, 2)[:, :kv]


def attention(q, k_pages, v_pages, table, kv_len, live, causal=True, window=0, sink=0, scale=None):
    """Attention over pages in 64 bits (all arguments on the host) -> out, lse, their bounds.

    With D channels and N tokens: a score is a sum of D products in fp32 (each adds 2^-23 of the sum of magnitudes), times a constant, less the
    running reference: off by at most e = scale sum |q k| (D + 32) 2^-23.  A weight is exp of it, off by exp(+-e) and 2^-21, and enters as two
    numbers of the type: 2^-16 of it (bf16), 2^-22 (binary16), in which a weight below 2^-14 of 2^7 times the row's largest one is off by 2^-32
    of that.  A product passes 2 (N / 32) + 64 fp32 sums.  So
        |out - exact| <= u |out| + (exp(2 e) - 1 + 2^-15 + (N / 16 + 64) 2^-23) E|v| + N 2^-31 max|v|  (the last for binary16),
        |lse - exact| <= e + 2^-20 (1 + |lse|) + (N / 16 + 64) 2^-23."""
    n, hq, m, d = q.shape
    H = k_pages.shape[0]
    g, scale = hq // H, 1 / math.sqrt(d) if scale is None else scale
    out, lse = torch.zeros(n, hq, m, d, dtype=torch.float64), torch.full((n, hq, m), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(n):
        kv, rows = int(kv_len[b]), int(live[b])
        if kv == 0 or rows == 0:
            continue
        see = sees(kv, rows, causal, window, sink)
        any_row = see.any(0)
        K, V = tokens_of(k_pages, table[b], kv).double(), tokens_of(v_pages, table[b], kv).double()
        K[:, ~any_row], V[:, ~any_row] = 0, 0
        sums = (kv / 16 + 64) * 2.0 ** -23
        for h in range(hq):
            k, v, x = K[h // g], V[h // g], q[b, h, :rows].double()
            s = (scale * (x @ k.T)).masked_fill(~see, -math.inf)
            e = scale * (x.abs() @ k.abs().T).masked_fill(~see, 0).amax(1) * (d + 32) * 2.0 ** -23
            z = torch.logsumexp(s, 1)
            ok = torch.isfinite(z)
            w = torch.where(ok[:, None], torch.exp(s - torch.where(ok, z, 0.0)[:, None]), 0.0)
            o = w @ v
            spread = w @ v.abs()
            t = HALF_STEP[q.dtype] * o.abs() + (torch.expm1(2 * e)[:, None] + 2.0 ** -15 + sums) * spread + TINY[q.dtype]
            if q.dtype is torch.float16:
                t = t + kv * 2.0 ** -31 * v.abs().amax()
            out[b, h, :rows], lse[b, h, :rows], tol[b, h, :rows] = o, z, torch.where(ok[:, None], t, 0.0)
            ltol[b, h, :rows] = torch.where(ok, e + 2.0 ** -20 * (1 + torch.where(ok, z, 0.0).abs()) + sums, 0.0)
    return out, lse, tol, ltol


def check_attention(got, lse, want):
    out, z, tol, ltol = want
    within(got, out, tol)
    dead = torch.isinf(z)
    lse = lse.cpu().double()
    assert torch.equal(torch.isinf(lse), dead) and (lse[dead] < 0).all()
    assert (got.cpu().double()[dead] == 0).all()
    off = (lse - z)[~dead].abs() - ltol[~dead]
    assert off.numel() == 0 or (off <= 0).all(), f"lse off by {float(off.max()):.3e} more than allowed"
