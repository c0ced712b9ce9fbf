"""What the paged operators' entry points refuse, without a GPU (every call fails before any launch, or has nothing to do)."""
import ctypes as C

import pytest
import torch

from paper_2602_02958_amd import binding as B

OK, NULL, BAD, UNSUPPORTED, WORKSPACE, ALIGN = 0, -1, -2, -3, -4, -5
FAKE = 0x1000                      # aligned, never read


def step(**kw):
    t = B.QvgTreeStep(n_seqs=2, group=1, n_nodes=4, table_pages=3, page_len=64, pool_pages=8, page_table=FAKE, kv_len=FAKE, q=FAKE,
                      q_stride_seq=512, q_stride_head=128, q_stride_node=128, k_new=FAKE, v_new=FAKE, new_stride_seq=512,
                      new_stride_head=128, new_stride_node=128, k_tail=FAKE, v_tail=FAKE, tail_stride_seq=1280, tail_stride_head=128,
                      tail_stride_token=128, tail_len=FAKE, tail_capacity=10, out=FAKE, out_stride_seq=512, out_stride_head=128,
                      out_stride_node=128)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def attn(t, pool=FAKE, scale=0.1, p=None, scratch=None, pools=None):
    pools = [pool] * 8 if pools is None else pools
    return B.lib().qvg_attn_tree(p or B.make_params(2, 16, 64, 1), None if t is None else C.byref(t), *pools, scale, scratch, 0, None)


def test_struct_layout_matches_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qvg.h")).read()
    body = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = body[body.index("typedef struct qvg_tree_step {"):body.index("} qvg_tree_step;")]
    names = []
    for decl in re.findall(r"(?:const )?(?:u?int\d+_t|void|float)\s+([^;]+);", body):
        names += [n.strip(" *") for n in decl.split(",")]
    assert names == [f[0] for f in B.QvgTreeStep._fields_]
    assert C.sizeof(B.QvgTreeStep) == 4 * 4 + 2 * 8 + 2 * 8 + 8 + 3 * 8 + 2 * 8 + 3 * 8 + 2 * 8 + 3 * 8 + 8 + 8 + 2 * 8 + 2 * 8 + 8 + 3 * 8 + 8


@pytest.mark.parametrize("kw", [
    dict(n_seqs=-1), dict(n_seqs=65536), dict(group=0), dict(n_nodes=-1), dict(table_pages=-1), dict(tail_capacity=-1), dict(reserved=1),
    dict(page_len=0), dict(page_len=1 << 31), dict(pool_pages=0), dict(pool_pages=1 << 31), dict(table_pages=1 << 20, page_len=1 << 11),
    dict(group=1 << 11, n_nodes=(1 << 9) + 1), dict(k_rope_f16=FAKE, rope_tokens=0), dict(table_pages=(1 << 31) - 1, page_len=1),
    dict(n_seqs=65535, group=1 << 10, n_nodes=1 << 10),
])
def test_attn_tree_sizes(kw):
    assert attn(step(**kw)) == BAD


@pytest.mark.parametrize("scale", [0.0, -1.0, float("inf"), float("nan")])
def test_attn_tree_scale(scale):
    assert attn(step(), scale=scale) == BAD


@pytest.mark.parametrize("name", ["q", "out", "k_new", "v_new", "page_table", "kv_len", "k_tail", "v_tail", "tail_len"])
def test_attn_tree_null(name):
    assert attn(step(**{name: None})) == NULL


@pytest.mark.parametrize("i", range(8))
def test_attn_tree_null_pool(i):
    assert attn(step(), pools=[None if j == i else FAKE for j in range(8)]) == NULL
    if i not in (1, 5):                                     # ids are bytes
        assert attn(step(), pools=[FAKE + 8 if j == i else FAKE for j in range(8)]) == ALIGN


@pytest.mark.parametrize("kw", [dict(q=FAKE + 8), dict(out=FAKE + 2), dict(k_new=FAKE + 4), dict(v_new=FAKE + 8), dict(k_tail=FAKE + 8),
                                dict(v_tail=FAKE + 8), dict(q_stride_node=132), dict(q_stride_head=4), dict(q_stride_seq=1),
                                dict(new_stride_node=130), dict(tail_stride_token=129), dict(out_stride_head=132), dict(page_table=FAKE + 2),
                                dict(kv_len=FAKE + 1), dict(mask=FAKE + 2), dict(nodes=FAKE + 3), dict(lse=FAKE + 2), dict(tail_len=FAKE + 2),
                                dict(k_rope_f16=FAKE + 8, rope_tokens=10)])
def test_attn_tree_alignment(kw):
    assert attn(step(**kw)) == ALIGN


def test_attn_tree_others():
    assert attn(None) == NULL
    assert attn(step(), scratch=FAKE + 8) == ALIGN
    assert attn(step(), p=B.make_params(2, 16, 64, 1, head_dim=64)) == UNSUPPORTED
    assert attn(step(), p=B.make_params(0, 16, 64, 1)) == BAD
    assert attn(step(n_seqs=0)) == OK and attn(step(n_nodes=0)) == OK
    assert attn(step(n_seqs=0, q=None, out=None), pool=None) == OK
    wide = B.make_params(2, 300, 64, 1)
    assert attn(step(), p=wide, pools=[FAKE, FAKE + 1] + [FAKE] * 6) == ALIGN


def test_attn_tree_scratch():
    p, out = B.make_params(2, 16, 64, 1), C.c_size_t(7)
    L = B.lib()
    assert L.qvg_attn_tree_scratch_bytes(p, C.byref(step(tail_capacity=0, table_pages=0)), C.byref(out)) == OK and out.value == 0
    assert L.qvg_attn_tree_scratch_bytes(p, C.byref(step(table_pages=1000)), C.byref(out)) == OK and out.value > 0
    assert L.qvg_attn_tree_scratch_bytes(p, C.byref(step(n_seqs=0)), C.byref(out)) == OK and out.value == 0
    assert L.qvg_attn_tree_scratch_bytes(p, C.byref(step()), None) == NULL
    assert L.qvg_attn_tree_scratch_bytes(p, None, C.byref(out)) == NULL
    assert L.qvg_attn_tree_scratch_bytes(p, C.byref(step(page_len=0)), C.byref(out)) == BAD


def test_tree_mask():
    f = B.lib().qvg_tree_mask
    assert f(-1, 4, FAKE, None, FAKE, None, None) == BAD
    assert f(1, -1, FAKE, None, FAKE, None, None) == BAD
    assert f(1, 1025, FAKE, None, FAKE, None, None) == BAD
    assert f(1 << 31, 4, FAKE, None, FAKE, None, None) == BAD
    assert f(1, 4, None, None, FAKE, None, None) == NULL
    assert f(1, 4, FAKE, None, None, None, None) == NULL
    for i in range(4):
        a = [FAKE + 2 if j == i else FAKE for j in range(4)]
        assert f(1, 4, *a, None) == ALIGN
    assert f(0, 4, None, None, None, None, None) == OK and f(3, 0, None, None, None, None, None) == OK


def keep(heads=2, d=128, n=3, nodes=5, k=FAKE, v=FAKE, ns=(640, 128, 128), path=FAKE, n_path=4, count=FAKE, kt=FAKE, vt=FAKE,
         ts=(1280, 128, 128), cap=10, length=FAKE, out=FAKE):
    return B.lib().qvg_keep_nodes(heads, d, n, nodes, k, v, *ns, path, n_path, count, kt, vt, *ts, cap, length, out, None)


def test_keep_nodes():
    for bad in (dict(heads=0), dict(heads=65536), dict(n=-1), dict(n=65536), dict(nodes=-1), dict(n_path=-1), dict(cap=-1),
                dict(cap=1 << 31), dict(n_path=1 << 21), dict(nodes=1 << 21), dict(n=65535, heads=65535, n_path=16)):
        assert keep(**bad) == BAD, bad
    assert keep(d=64) == UNSUPPORTED
    for null in ("k", "v", "path", "count", "kt", "vt", "length"):
        assert keep(**{null: None}) == NULL, null
    for off in (dict(k=FAKE + 8), dict(v=FAKE + 2), dict(kt=FAKE + 8), dict(vt=FAKE + 4), dict(ns=(640, 132, 128)), dict(ns=(641, 128, 128)),
                dict(ts=(1280, 128, 129)), dict(path=FAKE + 2), dict(count=FAKE + 1), dict(length=FAKE + 2), dict(out=FAKE + 3)):
        assert keep(**off) == ALIGN, off
    assert keep(n=0, count=None, length=None) == OK


def copy(pairs, page_len=64, src_pages=5, dst_pages=5, src=None, dst=None, p=None, n=None):
    ints = lambda v: (C.c_int32 * max(1, len(v)))(*v)
    src = [FAKE] * 4 if src is None else src
    dst = [2 * FAKE] * 4 if dst is None else dst
    return B.lib().qvg_copy_pages(p or B.make_params(2, 16, 64, 1), page_len, len(pairs) if n is None else n, ints([a for a, _ in pairs]),
                                  ints([b for _, b in pairs]), src_pages, *src, dst_pages, *dst, None)


def test_copy_pages():
    assert copy([]) == OK
    for bad in ([(5, 0)], [(-1, 0)], [(0, 5)], [(0, -1)], [(0, 1), (2, 1)], [(i % 5, i % 5) for i in range(6)]):
        assert copy(bad) == BAD, bad
    same = [FAKE] * 4
    # inside one pool no destination is a source
    for bad in ([(0, 0)], [(0, 1), (1, 2)], [(1, 2), (0, 1)]):
        assert copy(bad, dst=same) == BAD, bad
    assert copy([(0, 1)], page_len=0) == BAD and copy([(0, 1)], n=-1) == BAD
    assert copy([(0, 1)], dst_pages=0) == BAD and copy([(0, 0)], src_pages=0) == BAD
    for i in range(4):
        hole = [None if j == i else FAKE for j in range(4)]
        assert copy([(0, 1)], src=hole) == NULL and copy([(0, 1)], dst=hole) == NULL
        if i != 1:
            off = [FAKE + 8 if j == i else FAKE for j in range(4)]
            assert copy([(0, 1)], src=off) == ALIGN and copy([(0, 1)], dst=off) == ALIGN
    assert copy([(0, 1)], p=B.make_params(2, 16, 64, 1, head_dim=64)) == UNSUPPORTED


def test_the_binding_wants_tensors_of_the_gpu():
    x = torch.zeros(1, 2, 3, 128, dtype=torch.bfloat16)
    e = B.Encoded(torch.zeros(2, 1, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 8, dtype=torch.uint8),
                  torch.zeros(2, 8, 1, 32, dtype=torch.uint8), torch.zeros(2, 8, 1, 2, dtype=torch.float16), 8)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        B.attn_tree(x, e, e, None, None, x, x)
    with pytest.raises(TypeError):
        B.tree_mask(i[None])
    with pytest.raises(TypeError):
        B.keep_nodes(x, x, i[None], i, x, x, i)
    with pytest.raises((TypeError, ValueError)):
        B.copy_pages(e, [0], [0], into=e)
    with pytest.raises(ValueError, match="same length"):
        B.copy_pages(e, [0], [])
