"""Sizes at the ends of what the paged operators' interface takes."""
import ctypes as C
import math

import pytest
import torch

from test_tree_refusals import BAD, FAKE, OK, attn, step
from tree_util import D, Pool, reference

from paper_2602_02958_amd import binding as B

TOP = (1 << 31) - 1


def test_tiles_of_the_longest_tails_and_pages_are_counted():
    p, out = B.make_params(1, 16, 64, 1), C.c_size_t(7)
    need = []
    for capacity in (TOP - 31, TOP - 30, TOP):
        t = step(n_seqs=1, n_nodes=1, table_pages=0, tail_capacity=capacity)
        assert B.lib().qvg_attn_tree_scratch_bytes(p, C.byref(t), C.byref(out)) == OK
        need.append(out.value)
    assert need[0] > 0 and need == need[:1] * 3
    # tiles of one token each and a tail's 2^26: more than are counted in 32 bits
    assert attn(step(page_len=1, table_pages=TOP - 1024 - (1 << 26) + 8, tail_capacity=TOP)) == BAD


FORMS = [(dict(T=2), 1, False), (dict(T=1, fp8=True), 1, False), (dict(T=2), 20, False), (dict(T=1, B=16, S=4, fp8=True), 5, True),
         (dict(T=2), 70, False), (dict(T=2), 40, True), (dict(T=2, fp8=True), 3, False)]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,m,rope", FORMS, ids=str)
@pytest.mark.parametrize("divided", [True, False])
def test_a_page_of_all_the_tokens_that_a_number_counts(fmt, m, rope, divided):
    """A pool of one page whose first 100 tokens exist: a sequence reads no others."""
    n = 100
    pool = Pool(2, 1, n, K=16, seed=71, **fmt)
    g = torch.Generator().manual_seed(72)
    q, k, v = (torch.randn(1, 1, m, D, generator=g).to(torch.bfloat16) for _ in range(3))
    table = None
    if rope:
        ang = torch.rand(n, D // 2, generator=g, dtype=torch.float64) * 6.3
        table = torch.stack([ang.cos(), ang.sin()], -1).to(torch.float16)
    dev = [x.cuda() for x in (q, k, v)]
    sides = [pool.encoded(i, i + 1) for i in (0, 1)]
    ints = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(dev[0]), torch.empty(1, 1, m, device="cuda")
    rt = None if table is None else table.cuda()
    t = B.QvgTreeStep(n_seqs=1, group=1, n_nodes=m, table_pages=1, page_len=TOP, pool_pages=1, page_table=ints.data_ptr(),
                      kv_len=ints.data_ptr() + 4, q=dev[0].data_ptr(), q_stride_seq=m * D, q_stride_head=m * D, q_stride_node=D,
                      k_new=dev[1].data_ptr(), v_new=dev[2].data_ptr(), new_stride_seq=m * D, new_stride_head=m * D, new_stride_node=D,
                      out=out.data_ptr(), out_stride_seq=m * D, out_stride_head=m * D, out_stride_node=D, lse=lse.data_ptr(),
                      k_rope_f16=None if rt is None else rt.data_ptr(), rope_tokens=n if rope else 0)
    p = B.make_params(1, pool.K, pool.B, pool.T, bits=pool.bits, n_smooth_stages=pool.S,
                      scale_format=B.SCALE_E4M3 if pool.fp8 else B.SCALE_F16)
    need = C.c_size_t()
    assert B.lib().qvg_attn_tree_scratch_bytes(p, C.byref(t), C.byref(need)) == OK and need.value > 0
    scratch = torch.empty(need.value if divided else 0, dtype=torch.uint8, device="cuda")
    ptrs = [x.data_ptr() for e in sides for x in (e.centroids, e.ids, e.codes, e.scales)]
    assert B.lib().qvg_attn_tree(p, C.byref(t), *ptrs, 1 / math.sqrt(D), scratch.data_ptr() if divided else None, scratch.numel(),
                                 B._stream()) == OK
    none = torch.zeros(1, 1, 0, D, dtype=torch.bfloat16)
    want, z, tol, ltol = reference(q, pool, 1, [[0]], [n], k, v, none, none, [0], [m], torch.ones(1, m, m).tril().bool(), table)
    assert ((out.double().cpu() - want).abs() <= tol + 1e-30).all() and ((lse.double().cpu() - z).abs() <= ltol + 1e-30).all()


@pytest.mark.gpu
def test_a_tail_of_all_the_tokens_that_a_number_counts():
    """Every token of the tail is the same row (its stride is zero): the result is its V, the weights' sum 2^31 - 1 times one weight.
    Equal terms with V's 8 bits, 2^15 tiles to a wavefront: every partial sum is exact in fp32 but for the few that join."""
    g = torch.Generator().manual_seed(73)
    q, k, v, new = (torch.randn(1, 1, 1, D, generator=g).to(torch.bfloat16).cuda() for _ in range(4))
    pool = Pool(2, 1, 32, T=1, K=16, seed=74)
    out, lse = B.attn_tree(q, pool.encoded(0, 1), pool.encoded(1, 2), None, None, new, new, tail_k=k.expand(1, 1, TOP, D),
                           tail_v=v.expand(1, 1, TOP, D), tail_len=torch.tensor([TOP], dtype=torch.int32, device="cuda"),
                           mask=torch.zeros(1, 1, 1, dtype=torch.int32, device="cuda"), want_lse=True)
    s = float((q.double() * k.double()).sum()) / math.sqrt(D)
    assert torch.equal(out, v)                              # (far less off than half a step of bf16)
    # 128 products and the sum of weights in fp32, the logarithm: as tree_util.reference counts them
    e = 2.0 ** -20 * (float((q.double() * k.double()).abs().sum()) / math.sqrt(D) + 1 + abs(s + 31 * math.log(2)))
    assert abs(lse.item() - (s + math.log(TOP))) <= e


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_kept_tokens_of_a_tail_that_is_nearly_as_long_as_a_number_counts(in_place):
    """No path entry names a token, so no row is written; the lengths stop at the tail's end."""
    B_, M = 3, 40
    k = torch.zeros(B_, 1, 4, D, dtype=torch.bfloat16, device="cuda")
    row = torch.full((1, 1, 1, D), 3.0, dtype=torch.bfloat16, device="cuda")
    tail = row.expand(B_, 1, TOP, D)
    path = torch.full((B_, M), -1, dtype=torch.int32, device="cuda")
    keep = torch.tensor([M, 2, 3], dtype=torch.int32, device="cuda")
    lens = torch.tensor([TOP - 1, TOP - 2, TOP - 9], dtype=torch.int32, device="cuda")
    got = B.keep_nodes(k, k, path, keep, tail, tail, lens, out_len=lens if in_place else None)
    assert got.tolist() == [TOP, TOP, TOP - 6] and (row == 3.0).all()
