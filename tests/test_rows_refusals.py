"""What the rotary operators and the caches of 16-bit pages refuse, without a GPU (every call fails before any launch, or has nothing to
do)."""
import ctypes as C
import math
import os
import re

import pytest
import torch

from paper_2602_02958_amd import binding as B

OK, NULL, BAD, UNSUPPORTED, ALIGN = 0, -1, -2, -3, -5
FAKE = 0x1000                      # aligned, never read
BF16, F16, F32 = 0, 1, 2


def change(t, kw):
    for k, v in kw.items():
        assert hasattr(t, k)
        setattr(t, k, v)
    return t


def rotary(**kw):
    return change(B.QvgRotary(table=FAKE, type=F16, n_pairs=64, n_rows=100, half=0, positions=None), kw)


def cache(**kw):
    return change(B.QvgPageCache(type=BF16, n_seqs=2, n_heads=3, head_dim=128, table_pages=4, page_len=16, pool_pages=9, page_table=FAKE,
                                 kv_len=FAKE, k_pages=FAKE, v_pages=FAKE, stride_head=18432, stride_page=2048, stride_token=128), kw)


def step(**kw):
    return change(B.QvgPageStep(group=2, n_new=1, q=FAKE, q_stride_seq=768, q_stride_head=128, q_stride_token=128, causal=1, out=FAKE,
                                out_stride_seq=768, out_stride_head=128, out_stride_token=128), kw)


@pytest.mark.parametrize("name,struct", [("qvg_rotary", B.QvgRotary), ("qvg_page_cache", B.QvgPageCache), ("qvg_page_step", B.QvgPageStep)])
def test_struct_layouts_match_the_header(name, struct):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qvg.h")).read()
    body = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = body[body.index(f"typedef struct {name} {{"):body.index(f"}} {name};")]
    fields = []
    for kind, decl in re.findall(r"\n\s*(?:const )?(u?int\d+_t|void|float)\s+([^;]+);", body):
        fields += [(n.strip(" *"), 8 if "*" in n or kind == "int64_t" else 4) for n in decl.split(",")]
    assert [n for n, _ in fields] == [f[0] for f in struct._fields_]
    assert [size for _, size in fields] == [C.sizeof(f[1]) for f in struct._fields_]


# ---- tables -----------------------------------------------------------------------------------------------------
def table(n=5, pairs=64, freq=FAKE, first=0, positions=None, axes=1, axis=None, amplitude=1.0, kind=F16, out=FAKE):
    axis = None if axis is None else (C.c_int32 * len(axis))(*axis)
    return B.lib().qvg_rope_table(n, pairs, freq, first, positions, axes, axis, amplitude, kind, out, None)


def test_rope_table():
    for bad in (dict(n=-1), dict(n=1 << 31), dict(pairs=0), dict(pairs=257), dict(axes=0), dict(axes=9, positions=FAKE), dict(kind=BF16), dict(kind=3),
                dict(amplitude=math.nan), dict(amplitude=math.inf), dict(axes=2), dict(first=-1), dict(first=1 << 31), dict(first=(1 << 31) - 4),
                dict(pairs=2, axis=[0, 1]), dict(pairs=2, axes=2, positions=FAKE, axis=[0, 2]), dict(pairs=1, axis=[-1])):
        assert table(**bad) == BAD, bad
    assert table(freq=None) == NULL and table(out=None) == NULL
    for off in (dict(freq=FAKE + 4), dict(out=FAKE + 8), dict(positions=FAKE + 2)):
        assert table(**off) == ALIGN, off
    assert table(n=0, freq=None, out=None) == OK


# ---- rows -------------------------------------------------------------------------------------------------------
def rope(r=None, kind=BF16, n=2, heads=3, tokens=4, d=128, x=FAKE, xs=(1536, 512, 128), first=None, backward=0, out=2 * FAKE, os_=(1536, 512, 128)):
    return B.lib().qvg_rope(C.byref(rotary() if r is None else r), kind, n, heads, tokens, d, x, *xs, first, backward, out, *os_, None)


def test_rope():
    for bad in (dict(kind=3), dict(kind=-1), dict(n=-1), dict(heads=0), dict(heads=65536), dict(tokens=-1), dict(d=0), dict(d=12), dict(d=520),
                dict(backward=2), dict(n=1 << 16, tokens=1 << 15), dict(n=1 << 40), dict(out=FAKE, os_=(1536, 128, 512)),
                dict(r=rotary(type=BF16)), dict(r=rotary(n_pairs=0)), dict(r=rotary(n_pairs=65)), dict(r=rotary(n_rows=0)),
                dict(r=rotary(n_rows=1 << 31)), dict(r=rotary(half=2)), dict(r=rotary(reserved=1))):
        assert rope(**bad) == BAD, bad
    assert B.lib().qvg_rope(None, BF16, 1, 1, 1, 128, FAKE, 0, 0, 0, None, 0, FAKE, 0, 0, 0, None) == NULL
    for null in (dict(x=None), dict(out=None), dict(r=rotary(table=None))):
        assert rope(**null) == NULL, null
    for off in (dict(x=FAKE + 8), dict(out=FAKE + 2), dict(xs=(1536, 512, 132)), dict(os_=(1537, 512, 128)), dict(first=FAKE + 2),
                dict(r=rotary(table=FAKE + 2)), dict(r=rotary(table=FAKE + 4, type=F32)), dict(r=rotary(positions=FAKE + 1)),
                dict(kind=F32, xs=(1536, 512, 130))):
        assert rope(**off) == ALIGN, off
    assert rope(n=0, x=None, out=None) == OK and rope(tokens=0, x=None, out=None) == OK


# ---- appending --------------------------------------------------------------------------------------------------
def append(c=None, n=4, k=FAKE, v=FAKE, s=(1536, 512, 128), live=None, r=None, out=2 * FAKE):
    return B.lib().qvg_append_pages(C.byref(cache() if c is None else c), n, k, v, *s, live, None if r is None else C.byref(r), out, None)


BAD_CACHES = [dict(type=F32), dict(type=-1), dict(n_seqs=-1), dict(n_seqs=65536), dict(n_heads=0), dict(n_heads=65536), dict(head_dim=0),
              dict(table_pages=-1), dict(reserved=1), dict(page_len=0), dict(page_len=1 << 31), dict(pool_pages=0), dict(pool_pages=1 << 31),
              dict(table_pages=1 << 27), dict(table_pages=2, page_len=(1 << 29) + 1), dict(stride_token=-128), dict(stride_token=(1 << 24) + 8)]
OFF_CACHES = [dict(k_pages=FAKE + 8), dict(v_pages=FAKE + 2), dict(stride_head=4), dict(stride_page=2052), dict(stride_token=130),
              dict(page_table=FAKE + 2), dict(kv_len=FAKE + 1)]


def test_append_pages():
    for bad in BAD_CACHES + [dict(head_dim=20), dict(head_dim=1024)]:
        assert append(cache(**bad)) == BAD, bad
    for bad in (dict(n=-1), dict(n=1 << 31), dict(n=1 << 30), dict(r=rotary(n_pairs=65)), dict(r=rotary(type=5))):
        assert append(**bad) == BAD, bad
    assert B.lib().qvg_append_pages(None, 1, FAKE, FAKE, 0, 0, 0, None, None, None, None) == NULL
    for name in ("kv_len", "page_table", "k_pages", "v_pages"):
        assert append(cache(**{name: None})) == NULL, name
    for null in (dict(k=None), dict(v=None), dict(r=rotary(table=None))):
        assert append(**null) == NULL, null
    for off in OFF_CACHES:
        assert append(cache(**off)) == ALIGN, off
    for off in (dict(k=FAKE + 8), dict(v=FAKE + 4), dict(s=(1536, 516, 128)), dict(live=FAKE + 2), dict(out=FAKE + 3), dict(r=rotary(table=FAKE + 1))):
        assert append(**off) == ALIGN, off
    assert append(cache(n_seqs=0, kv_len=None), k=None) == OK


# ---- attention --------------------------------------------------------------------------------------------------
def attend(c=None, t=None, scale=0.1, scratch=None, size=0):
    return B.lib().qvg_attn_pages(C.byref(cache() if c is None else c), C.byref(step() if t is None else t), scale, scratch, size, None)


def test_attn_pages():
    for bad in BAD_CACHES:
        assert attend(cache(**bad)) == BAD, bad
    for bad in (dict(group=0), dict(n_new=-1), dict(group=1 << 11, n_new=(1 << 9) + 1), dict(causal=2), dict(causal=-1), dict(window=-1), dict(sink=-1),
                dict(reserved=1)):
        assert attend(t=step(**bad)) == BAD, bad
    assert attend(cache(n_seqs=4096, n_heads=4096)) == BAD and attend(cache(n_seqs=512, n_heads=128), step(group=1 << 10, n_new=8)) == BAD
    for scale in (0.0, -1.0, math.inf, math.nan, 3e38):
        assert attend(scale=scale) == BAD
    for d in (8, 32, 72, 80, 112, 160, 512):
        assert attend(cache(head_dim=d)) == UNSUPPORTED, d
    for name in ("kv_len", "page_table", "k_pages", "v_pages"):
        assert attend(cache(**{name: None})) == NULL, name
    assert attend(t=step(q=None)) == NULL and attend(t=step(out=None)) == NULL
    assert B.lib().qvg_attn_pages(None, C.byref(step()), 0.1, None, 0, None) == NULL
    assert B.lib().qvg_attn_pages(C.byref(cache()), None, 0.1, None, 0, None) == NULL
    for off in OFF_CACHES:
        assert attend(cache(**off)) == ALIGN, off
    for off in (dict(q=FAKE + 8), dict(out=FAKE + 2), dict(q_stride_head=132), dict(out_stride_seq=4), dict(n_live=FAKE + 2), dict(lse=FAKE + 1)):
        assert attend(t=step(**off)) == ALIGN, off
    assert attend(scratch=FAKE + 8) == ALIGN
    assert attend(cache(n_seqs=0, kv_len=None), step(q=None)) == OK and attend(t=step(n_new=0, q=None)) == OK


def test_scratch_bytes():
    out = C.c_size_t(7)

    def need(c=None, t=None):
        return B.lib().qvg_attn_pages_scratch_bytes(C.byref(c or cache()), C.byref(t or step()), C.byref(out))
    assert need() == OK and out.value == 0                                 # four pages of 16 tokens
    assert need(cache(table_pages=1000)) == OK and out.value > 0
    assert need(cache(table_pages=1000, n_seqs=0)) == OK and out.value == 0
    assert need(cache(table_pages=1000, n_seqs=300)) == OK and out.value == 0
    assert need(cache(table_pages=0)) == OK and out.value == 0
    assert need(cache(page_len=0)) == BAD and need(cache(head_dim=40)) == UNSUPPORTED
    assert B.lib().qvg_attn_pages_scratch_bytes(C.byref(cache()), C.byref(step()), None) == NULL
    assert B.lib().qvg_attn_pages_scratch_bytes(None, C.byref(step()), C.byref(out)) == NULL
    # never more than a fraction of what such a call's cache takes, whatever the heads and rows
    for seqs in (1, 3, 16, 64, 255, 256):
        for heads in (1, 8, 40, 200, 500):
            for rows in (1, 16, 17, 64):
                for d in (64, 128, 256):
                    assert need(cache(n_seqs=seqs, n_heads=heads, head_dim=d, table_pages=4096), step(group=rows)) == OK
                    assert out.value <= 160 << 20, (seqs, heads, rows, d, out.value)


# ---- the binding --------------------------------------------------------------------------------------------------
def test_frequencies():
    f, a = B.rope_frequencies(8, base=16.0, device="cpu")
    assert a == 1.0 and f.dtype is torch.float64 and f.tolist() == [1.0, 0.5, 0.25, 0.125]
    assert torch.equal(B.rope_frequencies(8, base=16.0, scaling="linear", factor=4.0, device="cpu")[0], f / 4)
    g, a = B.rope_frequencies(8, base=16.0, scaling="base", factor=8.0, device="cpu")
    assert a == 1.0 and g[0] == 1.0 and abs(float(g[3] - f[3] / 8)) < 1e-15
    # 200 places: 31.8, 15.9, 8.0 and 4.0 turns
    g, a = B.rope_frequencies(8, base=16.0, scaling="bands", factor=4.0, trained=200, low=5.0, high=20.0, device="cpu")
    keep = [1.0, (200 * 0.5 / (2 * math.pi) - 5) / 15, (200 * 0.25 / (2 * math.pi) - 5) / 15, 0.0]
    assert torch.allclose(g, f * torch.tensor([k + (1 - k) / 4 for k in keep], dtype=torch.float64), rtol=1e-14)
    assert abs(a - (0.1 * math.log(4) + 1)) < 1e-15
    for bad in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=8, base=0.0), dict(rotary_dim=8, factor=0.5), dict(rotary_dim=8, scaling="x"),
                dict(rotary_dim=8, base=math.inf), dict(rotary_dim=2, scaling="base", factor=2.0), dict(rotary_dim=8, scaling="bands", factor=2.0),
                dict(rotary_dim=8, scaling="bands", factor=2.0, trained=100, low=3.0, high=3.0)):
        with pytest.raises(ValueError):
            B.rope_frequencies(device="cpu", **bad)


def test_the_binding_wants_tensors_of_the_gpu():
    x, pages = torch.zeros(1, 2, 3, 128, dtype=torch.bfloat16), torch.zeros(2, 4, 8, 128, dtype=torch.bfloat16)
    t, i = torch.zeros(9, 64, 2, dtype=torch.float16), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: B.rope(x, t), lambda: B.rope_table(3, torch.zeros(4, dtype=torch.float64)), lambda: B.append_pages(x, x, pages, pages, i[None], i),
                 lambda: B.attn_pages(x, pages, pages, i[None], i)):
        with pytest.raises(TypeError):
            call()


class On(torch.Tensor):
    """A host tensor that says it lies on GPU number .at."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.at


def on(t, at=0):
    t = t.as_subclass(On)
    t.at = at
    return t


@pytest.fixture
def device_zero(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)

    def launched(*a):
        raise AssertionError("the call went on")
    monkeypatch.setattr(B, "_stream", launched)


def args(at=None):
    """Arguments of each kind, the one named `at` on another device."""
    a = dict(x=torch.zeros(1, 2, 3, 128, dtype=torch.bfloat16), v=torch.zeros(1, 2, 3, 128, dtype=torch.bfloat16),
             k_pages=torch.zeros(2, 4, 8, 128, dtype=torch.bfloat16), v_pages=torch.zeros(2, 4, 8, 128, dtype=torch.bfloat16),
             table=torch.zeros(9, 64, 2, dtype=torch.float16), positions=torch.zeros(1, 3, dtype=torch.int32),
             first=torch.zeros(1, dtype=torch.int32), page_table=torch.zeros(1, 5, dtype=torch.int32), kv_len=torch.zeros(1, dtype=torch.int32),
             n_new=torch.zeros(1, dtype=torch.int32), out=torch.zeros(1, 2, 3, 128, dtype=torch.bfloat16), len=torch.zeros(1, dtype=torch.int32),
             scratch=torch.zeros(0, dtype=torch.uint8), freq=torch.zeros(64, dtype=torch.float64), places=torch.zeros(9, 1, dtype=torch.int32))
    return {k: on(t, 1 if k == at else 0) for k, t in a.items()}


CALLS = {
    "rope": (lambda a: B.rope(a["x"], a["table"], positions=a["positions"], out=a["out"]), ["x", "table", "positions", "out"]),
    "rope first": (lambda a: B.rope(a["x"], a["table"], first=a["first"], out=a["out"]), ["first"]),
    "table": (lambda a: B.rope_table(9, a["freq"], positions=a["places"], out=a["table"]), ["freq", "places", "table"]),
    "append": (lambda a: B.append_pages(a["x"], a["v"], a["k_pages"], a["v_pages"], a["page_table"], a["kv_len"], a["n_new"], a["table"], a["positions"],
                                        out_len=a["len"]),
               ["x", "v", "k_pages", "v_pages", "page_table", "kv_len", "n_new", "table", "positions", "len"]),
    "attend": (lambda a: B.attn_pages(a["x"], a["k_pages"], a["v_pages"], a["page_table"], a["kv_len"], a["n_new"], out=a["out"], scratch=a["scratch"]),
               ["x", "k_pages", "v_pages", "page_table", "kv_len", "n_new", "out", "scratch"]),
}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_device_are_refused(name, device_zero):
    call, who = CALLS[name]
    for at in who:
        with pytest.raises(ValueError, match="current device"):
            call(args(at))
    with pytest.raises(AssertionError, match="went on"):
        call(args())


WRONG = [  # call, argument, what it is instead
    ("rope", "x", lambda t: t[0]), ("rope", "x", lambda t: t.double()), ("rope", "x", lambda t: t[..., ::2]), ("rope", "table", lambda t: t.double()),
    ("rope", "table", lambda t: t[:, ::2]), ("rope", "table", lambda t: t[:0]), ("rope", "positions", lambda t: t.long()),
    ("rope", "positions", lambda t: t[:, :2]), ("rope", "out", lambda t: t.half()), ("rope", "out", lambda t: t[:, :1]),
    ("rope", "out", lambda t: t[:, :1].expand(1, 2, 3, 128)), ("rope first", "first", lambda t: t[None]),
    ("table", "freq", lambda t: t.float()), ("table", "places", lambda t: t[:, 0]), ("table", "places", lambda t: t[:5]), ("table", "table", lambda t: t.float()),
    ("table", "table", lambda t: t[:5]), ("append", "x", lambda t: t.half()), ("append", "v", lambda t: t[:, :, :2]),
    ("append", "v", lambda t: torch.zeros(1, 3, 2, 128, dtype=torch.bfloat16).transpose(1, 2)), ("append", "k_pages", lambda t: t.float()),
    ("append", "k_pages", lambda t: t[:1]), ("append", "v_pages", lambda t: t[:, :, :4]), ("append", "v_pages", lambda t: t.half()),
    ("append", "v_pages", lambda t: torch.zeros(2, 8, 4, 128, dtype=torch.bfloat16).transpose(1, 2)), ("append", "page_table", lambda t: t[0]),
    ("append", "page_table", lambda t: t.long()), ("append", "page_table", lambda t: t[:, ::2]), ("append", "kv_len", lambda t: t[None]),
    ("append", "n_new", lambda t: t.float()), ("append", "len", lambda t: t.long()), ("append", "positions", lambda t: t[0]),
    ("attend", "x", lambda t: t[:, :1]), ("attend", "x", lambda t: t[..., :64]), ("attend", "x", lambda t: t.half()), ("attend", "kv_len", lambda t: t[:0]),
    ("attend", "out", lambda t: t[:, :, :2]), ("attend", "scratch", lambda t: t.int()), ("attend", "n_new", lambda t: t[None]),
]


@pytest.mark.parametrize("i", range(len(WRONG)))
def test_arguments_of_other_shapes_and_types_are_refused(i, device_zero):
    name, at, other = WRONG[i]
    a = args()
    a[at] = on(other(a[at].as_subclass(torch.Tensor)))
    with pytest.raises((TypeError, ValueError)):
        CALLS[name][0](a)


def test_pages_that_are_written_lie_in_places_of_their_own(device_zero):
    a = args()
    for at in ("k_pages", "v_pages"):
        a[at] = on(torch.zeros(1, 4, 8, 128, dtype=torch.bfloat16).expand(2, 4, 8, 128))
    with pytest.raises(ValueError, match="places of their own"):
        CALLS["append"][0](a)
    with pytest.raises(AssertionError, match="went on"):                   # (heads that share their pages are read)
        CALLS["attend"][0](a)


def test_what_says_a_thing_twice_or_not_at_all(device_zero):
    a = args()
    with pytest.raises(ValueError, match="both"):
        B.rope(a["x"], a["table"], positions=a["positions"], first=a["first"])
    with pytest.raises(ValueError, match="not turned"):
        B.append_pages(a["x"], a["v"], a["k_pages"], a["v_pages"], a["page_table"], a["kv_len"], positions=a["positions"])
    with pytest.raises(ValueError, match="window"):
        B.attn_pages(a["x"], a["k_pages"], a["v_pages"], a["page_table"], a["kv_len"], window=0, out=a["out"], scratch=a["scratch"])
    with pytest.raises(ValueError, match="axes of 64"):
        B.rope_table(9, a["freq"], positions=a["places"], axis=[0] * 63, out=a["table"])
    with pytest.raises(OverflowError):
        B.rope_table(9, a["freq"], positions=a["places"], axis=[1 << 40] * 64, out=a["table"])
    with pytest.raises(TypeError):
        B.rope_table(9, a["freq"], dtype=torch.bfloat16)
    x = on(torch.zeros(1, 4, 4, 128, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="strides"):
        B.rope(x, a["table"], out=on(x.as_subclass(torch.Tensor).transpose(1, 2)))


def test_a_paged_cache_turns_the_keys_it_is_given_with_a_table(monkeypatch):
    monkeypatch.setattr(B, "_check", lambda *a: None)
    monkeypatch.setattr(B, "_here", lambda *a: None)
    init = torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    make = lambda **kw: B.PagedCache(1, 2, 6, 8, 4, 20, 8, 64, 1, init, device="cpu", **kw)            # noqa: E731
    pre, plain = make(pre_rope=True), make()
    seen = []

    def turned(x, table, first=None):
        seen.append((x.shape, first.tolist()))
        return x + 1
    monkeypatch.setattr(B, "rope", turned)
    t, s = pre.open(), plain.open()
    table, kv = torch.zeros(40, 64, 2, dtype=torch.float16), torch.randn(2, 3, 128).to(torch.bfloat16)
    for n in range(2):
        pre.append(t, kv, k_rope=table)
    assert seen == [((1, 1, 3, 128), [0]), ((1, 1, 3, 128), [3])]
    assert torch.equal(pre.tail[t, :2, 3:6], kv) and torch.equal(pre.tail[t, 2:, 3:6], kv[:1] + 1)
    for cache, seq, kw in ((plain, s, dict(k_rope=table)), (pre, t, dict(k_rope=table, k_rotated=kv[:1])), (pre, t, dict(k_rope=table[:, :32])),
                           (pre, 1, dict(k_rope=table))):
        with pytest.raises(ValueError):
            cache.append(seq, kv, **kw)
    assert pre.length(t) == 6
