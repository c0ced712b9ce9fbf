"""attn_tree on scores of any finite magnitude: where fp32 holds no fraction of a score any more, equal scores still weigh alike and the
weights of others follow the scores' differences."""
import math

import pytest
import torch

from tree_util import D, Pool

pytestmark = pytest.mark.gpu
B = pytest.importorskip("paper_2602_02958_amd.binding")

# log2(e) times this is 1 in fp32: scores in powers of two are what the products give
LN2 = 0.693147182464599609375
FORMS = [(dict(T=1, fp8=True), 1, 1), (dict(T=2), 1, 5), (dict(T=2), 2, 12), (dict(T=2), 5, 16), (dict(T=1, B=16, S=4, fp8=True), 1, 2),
         (dict(T=2, fp8=True), 1, 3), (dict(T=1, bits=4, fp8=True), 2, 14)]


def step(fmt, g, m, keys, values, n_page, q, scale, where, rope=False):
    """keys, values [n, D]: n tokens in pages of n_page (every token its own centroid), or in the tail.  All rows of q are alike."""
    n = keys.shape[0]
    dev = lambda t: t.to(torch.bfloat16).cuda()                                                             # noqa: E731
    K = n_page if where == "pages" else 16
    pages = n // n_page if where == "pages" else 1
    sides = []
    for x in (keys, values):
        pool = Pool(1, pages, n_page, K=K, seed=81, **fmt)
        if where == "pages":
            pool.cent[:] = 0
            pool.cent[0, :, 0] = x.view(pages, n_page, D).to(torch.bfloat16)
            pool.ids[:] = 0
            pool.ids[0, :, 0] = torch.arange(n) % n_page    # (other stages: row 0, which the first one's token 0 has alone)
            pool.cent[0, :, 1:] = 0
            pool.codes[:] = 0
        sides.append(pool.encoded(0, 1))
    row = dev(q).expand(1, g, m, D).contiguous()
    nothing = torch.zeros(1, 1, m, D, dtype=torch.bfloat16, device="cuda")
    kw = dict(mask=torch.zeros(1, m, -(-m // 32), dtype=torch.int32, device="cuda"), softmax_scale=scale, want_lse=True)
    if where == "pages":
        if rope:                                           # (turned by nothing: the form that rotates)
            table = torch.zeros(n, D // 2, 2, dtype=torch.float16, device="cuda")
            table[..., 0] = 1
            kw["k_rope"] = table
        return B.attn_tree(row, *sides, torch.arange(pages, dtype=torch.int32, device="cuda")[None],
                           torch.tensor([n], dtype=torch.int32, device="cuda"), nothing, nothing, **kw)
    return B.attn_tree(row, *sides, None, None, nothing, nothing, tail_k=dev(keys)[None, None], tail_v=dev(values)[None, None],
                       tail_len=torch.tensor([n], dtype=torch.int32, device="cuda"), **kw)


def close(got, want, values):
    """Weights of 11 bits of values rounded to 11 bits (2^-10 of the largest), the result's rounding to bf16."""
    err = (got[0].double().cpu() - want).abs()
    assert (err <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * values.abs().max()).all(), err.max()


@pytest.mark.parametrize("where,rope", [("pages", False), ("pages", True), ("tail", False)])
@pytest.mark.parametrize("fmt,g,m", FORMS, ids=str)
@pytest.mark.parametrize("top", [0, 14, 23, 24, 27, 28, 40, 100, 125])
def test_equal_scores_weigh_alike(fmt, g, m, where, rope, top):
    """256 tokens of one key, whose score is 0.12 times 2^top (times a scale of all bits): the mean of their values."""
    gen = torch.Generator().manual_seed(82)
    values = torch.randn(256, D, generator=gen).to(torch.bfloat16)
    key, q = torch.zeros(D), torch.zeros(D)
    key[3], q[3] = 1.3671875, 2.0 ** top
    scale = 1.0 / math.sqrt(D)
    got = step(fmt, g, m, key.expand(256, D).contiguous(), values, 64, q, scale, where, rope)
    close(got, values.double().mean(0), values)
    s = 1.3671875 * 2.0 ** top * scale
    assert torch.allclose(got[1].double().cpu(), torch.tensor(s + math.log(256), dtype=torch.float64), rtol=2.0 ** -21, atol=2.0 ** -20)


@pytest.mark.parametrize("where,rope", [("pages", False), ("pages", True), ("tail", False)])
@pytest.mark.parametrize("fmt,g,m", FORMS, ids=str)
@pytest.mark.parametrize("top,apart", [(26, 8), (25, 8), (24, 4), (26, 64), (20, 13), (26, -8), (40, 1 << 20), (100, -(1 << 80)), (125, 1 << 104)])
def test_weights_follow_the_differences(fmt, g, m, where, rope, top, apart):
    """128 tokens of score 2^top (in powers of two), then 128 of 2^top + apart: fp32 holds both."""
    gen = torch.Generator().manual_seed(83)
    values = torch.randn(256, D, generator=gen).to(torch.bfloat16)
    key, q = torch.zeros(256, D), torch.zeros(D)
    key[:, 5], q[5] = 2.0 ** (top - top // 2 if top < 28 else 14), 2.0 ** (top // 2 if top < 28 else top - 14)
    key[128:, 9], q[9] = float(apart) / 2.0 ** math.floor(math.log2(abs(apart))), 2.0 ** math.floor(math.log2(abs(apart)))
    got = step(fmt, g, m, key, values, 128, q, LN2, where, rope)
    first, second = values[:128].double().mean(0), values[128:].double().mean(0)
    w = 0.0 if apart < -60 else math.inf if apart > 60 else 2.0 ** apart
    want = second if math.isinf(w) else (first + w * second) / (1 + w)
    close(got, want, values)
