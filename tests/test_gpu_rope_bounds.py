"""The bounds that the rotary operators promise, held as tightly as they are promised: a far place's angle, and places on which scores depend."""
import math
from decimal import Decimal
from fractions import Fraction

import pytest
import torch

from paper_2602_02958_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, F32 = torch.float16, torch.float32


TWO_PI = Fraction(Decimal("6.28318530717958647692528676655900576839433879875021164194989"))


def cos_sin_of(place, f):
    """Of place * f, taken exactly and reduced by a 2 pi of 60 digits before 64 bits round it."""
    out = torch.empty(len(place), len(f), 2, dtype=torch.float64)
    for j, x in enumerate(f):
        for i, p in enumerate(place):
            a = Fraction(p) * Fraction(x)
            r = float(a - round(a / TWO_PI) * TWO_PI)
            out[i, j, 0], out[i, j, 1] = math.cos(r), math.sin(r)
    return out


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("pairs,base", [(64, 10000.0), (7, 500.0), (30, 1e6)])
def test_far_places_lose_2_to_the_minus_51_of_their_angle(pairs, base, dtype):
    """Three 64-bit roundings (2 / pi, its product with the frequency, that with the place) are 2^-51 of the angle, in radians; a quarter turn's
    fraction is rounded to 32 bits (2^-25 of half of one) and times pi / 2 (2^-24 of pi / 4), the polynomials leave 2^-29 and their last
    steps 2^-23; the amplitude is 1."""
    f, _ = B.rope_frequencies(2 * pairs, base=base, device=DEV)
    place = [0, 1, 2, 4095, 37439, 748799, 12345678, (1 << 26) + 1, (1 << 30) - 3, (1 << 31) - 2, (1 << 31) - 1, -1, -(1 << 31), -748800]
    pos = torch.tensor(place, dtype=torch.int64).to(torch.int32)[:, None].contiguous().to(DEV)
    got = B.rope_table(len(place), f, positions=pos, dtype=dtype).cpu().double()
    want = cos_sin_of(place, f.tolist())
    angle = (torch.tensor(place, dtype=torch.float64)[:, None] * f.cpu()).abs()
    tol = angle * 2.0 ** -51 + math.pi / 2 * 2.0 ** -26 + math.pi / 4 * 2.0 ** -23 + 2.0 ** -29 + 2.0 ** -23 + 2.0 ** -49
    tol = tol[..., None] + (2.0 ** -12 + 2.0 ** -25 if dtype is F16 else 0.0)
    far = (got - want).abs() - tol
    assert (far <= 0).all(), f"off by {float(far.max()):.3e} more than allowed at {int(far.argmax())}"


def test_scores_depend_on_the_distance_of_places_and_on_nothing_less():
    """Equal distances give equal results, within their roundings; keys moved on alone, or rows that are not turned, others by far more."""
    d, n = 128, 24
    f, _ = B.rope_frequencies(d, device=DEV)
    rotary = B.rope_table(5000, f, dtype=F32)
    q, kn, vn = (torch.randn(1, 1, n, d, generator=torch.Generator().manual_seed(i)).to(F16).to(DEV) for i in (1, 2, 3))

    def attend(q_shift, k_shift):
        k, v = B.alloc_pages(1, 2, 16, d, F16, DEV)
        table, lens = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        at = torch.arange(n, dtype=torch.int32, device=DEV)[None]
        lens = B.append_pages(kn, vn, k, v, table, lens, k_rope=None if k_shift is None else rotary, positions=None if k_shift is None else at + k_shift)
        turned = q if q_shift is None else B.rope(q, rotary, positions=at + q_shift)
        return B.attn_pages(turned, k, v, table, lens).double()

    base = attend(0, 0)
    # keys and queries are rounded once more after the turn: a score, a sum of 128 products of sizes |q_c k_c|, by 2 x 2^-11 of them; the
    # sum of |q_c| |k_c| over the scale is at most |q| |k| / sqrt(d) < 1.15^2 sqrt(d) < 15.  A weight by exp of twice that, at either shift;
    # outputs, means of |v| < 4, once more by 2^-11
    assert max(float(t.float().norm(dim=-1).max()) for t in (q, kn)) < 1.15 * math.sqrt(d) and vn.abs().max() < 4
    same = 4 * (math.expm1(2 * 15 * 2 * 2.0 ** -11) * 2 + 2 * 2.0 ** -11)
    assert (base - attend(1000, 1000)).abs().max() <= same
    for q_shift, k_shift in ((1000, 0), (0, 1000), (None, None), (0, None), (None, 0)):
        assert (base - attend(q_shift, k_shift)).abs().max() > 2 * same, (q_shift, k_shift)
