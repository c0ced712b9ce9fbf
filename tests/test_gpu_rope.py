"""Rotary tables and turned rows against their definitions in 64 bits."""
import math

import pytest
import torch

from paper_2602_02958_amd import binding as B
from rows_util import turned, within

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- tables ---------------------------------------------------------------------------------------------------
def table_bound(angle, dtype, amplitude=1.0):
    """An angle in turns is off by 2^-51 of itself (two 64-bit roundings) and then by a rounding to 2^-25 turns; sine and cosine by 2^-22."""
    err = angle.abs() * 2.0 ** -51 * 2 * math.pi + 2 * math.pi * 2.0 ** -25 + 2.0 ** -22
    return amplitude * err + (2.0 ** -11 * amplitude + 2.0 ** -25 if dtype is F16 else 2.0 ** -23 * amplitude)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("n,pairs,first", [(1, 1, 0), (3, 64, 0), (1000, 64, 747000), (257, 30, 5), (70, 256, 100), (5, 7, (1 << 31) - 5),
                                           (2100, 128, 12345678)])
def test_tables_of_places(n, pairs, first, dtype):
    f, amp = B.rope_frequencies(2 * pairs, device=DEV)
    assert amp == 1.0
    got = B.rope_table(n, f, first=first, dtype=dtype)
    ang = (torch.arange(n, dtype=torch.float64) + first)[:, None] * f.cpu()
    want = torch.stack([ang.cos(), ang.sin()], -1)
    within(got, want, table_bound(ang, dtype)[..., None].expand_as(want))


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("n,pairs,axes", [(1, 3, 3), (1000, 64, 3), (333, 22, 1), (64, 256, 8)])
def test_tables_of_axes(n, pairs, axes, dtype):
    pos = torch.randint(-50, 800000, (n, axes), generator=gen(1), dtype=torch.int32)
    axis = [(p * 7 + 3) % axes for p in range(pairs)]
    f, amp = B.rope_frequencies(2 * pairs, base=500.0, scaling="bands", factor=8.0, trained=4096, device=DEV)
    got = B.rope_table(n, f, positions=pos.to(DEV), axis=axis, amplitude=amp, dtype=dtype)
    ang = pos[:, axis].double() * f.cpu()
    want = amp * torch.stack([ang.cos(), ang.sin()], -1)
    within(got, want, table_bound(ang, dtype, amp)[..., None].expand_as(want))


def test_a_table_of_no_rows_and_a_given_place():
    f, _ = B.rope_frequencies(128, device=DEV)
    assert B.rope_table(0, f).shape == (0, 64, 2)
    out = torch.empty(9, 64, 2, dtype=F32, device=DEV)
    assert B.rope_table(9, f, dtype=F32, out=out) is out
    assert torch.equal(out, B.rope_table(9, f, dtype=F32))


# ---- rows -------------------------------------------------------------------------------------------------------
def rows(shape, dtype, seed, order="bhnd"):
    """Rows [B, H, N, d], as they are or as a view of [B, N, H, d]."""
    n, h, m, d = shape
    if order == "bhnd":
        return torch.randn(shape, generator=gen(seed)).to(dtype)
    return torch.randn(n, m, h, d, generator=gen(seed)).to(dtype).transpose(1, 2)


def table(n, pairs, dtype, seed):
    ang = torch.rand(n, pairs, generator=gen(seed), dtype=torch.float64) * 50 - 25
    return (torch.stack([ang.cos(), ang.sin()], -1) * 1.2).to(dtype)


SHAPES = [  # B, H, N, d, pairs, order
    (1, 1, 1, 128, 64, "bhnd"), (2, 3, 5, 128, 64, "bnhd"), (3, 5, 37, 64, 32, "bnhd"), (1, 12, 300, 96, 32, "bhnd"), (2, 1, 17, 8, 4, "bhnd"),
    (1, 2, 9, 512, 256, "bhnd"), (2, 7, 33, 192, 20, "bnhd"), (1, 4, 11, 80, 3, "bhnd"), (4, 2, 3, 256, 65, "bnhd"), (1, 6, 1000, 40, 8, "bnhd"),
    (1, 1, 3, 16, 1, "bhnd"), (1, 9, 1200, 128, 64, "bnhd"), (1, 3, 5, 512, 250, "bhnd"),
]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("dtype,tdtype", [(BF, F16), (F16, F32), (F32, F32), (BF, F32), (F32, F16)])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows(shape, dtype, tdtype, half):
    *bhnd, pairs, order = shape
    n, h, m, d = bhnd
    x, t = rows(bhnd, dtype, 3, order), table(64, pairs, tdtype, 4)
    pos = torch.randint(-3, 70, (n, m), generator=gen(5), dtype=torch.int32)
    want, tol = turned(x, t[pos.long().clamp(0, 63)][:, None], half)
    xd = x.to(DEV)
    assert xd.stride() == x.stride()
    got = B.rope(xd, t.to(DEV), positions=pos.to(DEV), half=half)
    within(got, want, tol)
    assert torch.equal(xd.cpu(), x)
    # the gradient, and in place
    want, tol = turned(x, t[pos.long().clamp(0, 63)][:, None], half, backward=True)
    assert B.rope(xd, t.to(DEV), positions=pos.to(DEV), half=half, backward=True, out=xd) is xd
    within(xd, want, tol)


@pytest.mark.parametrize("half", [False, True])
def test_many_rows_of_many_heads(half):
    # (several heads to a thread)
    x, t = rows((3, 21, 1500, 128), BF, 6, "bnhd"), table(2000, 48, F16, 7)
    first = torch.tensor([0, 499, 1990], dtype=torch.int32)
    at = (first.long()[:, None] + torch.arange(1500)).clamp(max=1999)
    want, tol = turned(x, t[at][:, None], half)
    within(B.rope(x.to(DEV), t.to(DEV), first=first.to(DEV), half=half), want, tol)


def test_places_without_positions():
    x, t = rows((2, 3, 10, 128), F32, 8), table(10, 64, F32, 9)
    want, tol = turned(x, t[None, None])
    within(B.rope(x.to(DEV), t.to(DEV)), want, tol)
    first = torch.tensor([-4, 1 << 30], dtype=torch.int32)
    at = (first.long()[:, None] + torch.arange(10)).clamp(0, 9)
    want, tol = turned(x, t[at][:, None])
    within(B.rope(x.to(DEV), t.to(DEV), first=first.to(DEV)), want, tol)


def test_a_table_that_starts_between_16_byte_places_and_strided_outputs():
    x = rows((2, 2, 6, 128), BF, 10)
    whole = torch.zeros(7 * 128 + 2, dtype=F16, device=DEV)
    t = table(7, 64, F16, 11)
    shifted = whole[2:].view(7, 64, 2)
    shifted.copy_(t)
    assert shifted.data_ptr() % 16 == 4
    out = torch.full((2, 6, 2, 136), 7.0, dtype=BF, device=DEV)
    view = out[..., :128].transpose(1, 2)
    want, tol = turned(x, t[:6][None, None])
    assert B.rope(x.to(DEV), shifted, out=view) is view
    within(view, want, tol)
    assert (out[..., 128:] == 7).all()                       # nothing behind the rows


@pytest.mark.parametrize("pairs", [32, 30, 29, 1])
@pytest.mark.parametrize("dtype", [BF, F16, F32])
def test_channels_behind_the_pairs_stay_bit_for_bit_even_no_numbers(dtype, pairs):
    x = rows((1, 2, 3, 128), dtype, 12)
    whole = {2: torch.int16, 4: torch.int32}[x.element_size()]
    bits = x.view(whole)
    top = -1 if whole is torch.int16 else -(1 << 20)
    bits[..., 2 * pairs:] = torch.arange(128 - 2 * pairs, dtype=whole) + (top - 200)            # no numbers, of many kinds
    x[..., 100] = math.inf
    for half in (False, True):
        for out in (None, x.to(DEV)):
            xd = x.to(DEV) if out is None else out
            got = B.rope(xd, table(3, pairs, F16, 13).to(DEV), half=half, out=out).cpu()
            assert torch.equal(got.view(whole)[..., 2 * pairs:], bits[..., 2 * pairs:])
            assert torch.isfinite(got[..., :2 * pairs].float()).all()


def test_gradient_against_differences():
    """d/dx of a weighted sum of turned rows, by central differences in 64 bits of the definition, is the backward form of the weights."""
    x, t = rows((1, 2, 3, 16), F32, 14), table(3, 6, F32, 15)
    w = rows((1, 2, 3, 16), F32, 16)
    for half in (False, True):
        got = B.rope(w.to(DEV), t.to(DEV), half=half, backward=True).cpu().double()
        step, xd = 1e-4, x.double()
        for i in range(0, x.numel(), 5):
            e = torch.zeros(x.numel(), dtype=torch.float64)
            e[i] = step
            e = e.view(x.shape)
            up, down = (((turned(y, t[None, None], half)[0]) * w.double()).sum() for y in ((xd + e).to(torch.float64), xd - e))
            diff = float(up - down) / (2 * step)
            # (linear: the difference is exact but for 64-bit roundings over the step)
            assert abs(diff - float(got.flatten()[i])) <= 2.0 ** -21 * 3 + 1e-10


def test_a_row_turned_and_turned_back():
    x = rows((2, 4, 50, 128), F32, 17).to(DEV)
    f, _ = B.rope_frequencies(128, device=DEV)
    t = B.rope_table(50, f, dtype=F32)
    back = B.rope(B.rope(x, t), t, backward=True)
    # cos^2 + sin^2 of stored numbers is 1 within 2^-20 (each off by 2^-21 at most), and two turns round twice
    assert ((back - x).abs() <= 2.0 ** -18 * x.abs().amax()).all()


def test_on_another_stream_and_in_a_graph():
    x, t = rows((2, 4, 9, 128), BF, 18).to(DEV), table(9, 64, F16, 19).to(DEV)
    want = B.rope(x, t)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = B.rope(x, t)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    f, _ = B.rope_frequencies(128, device=DEV)
    tab, out = torch.empty(9, 64, 2, dtype=F16, device=DEV), torch.empty_like(x)
    B.rope_table(9, f, out=tab)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.rope_table(9, f, axis=[0] * 64, out=tab)
        B.rope(x, tab, out=out)
    for i in range(3):
        x.copy_(rows((2, 4, 9, 128), BF, 20 + i))
        tab.zero_(), out.zero_()
        g.replay()
        assert torch.equal(out, B.rope(x, B.rope_table(9, f)))
        torch.cuda.synchronize()
