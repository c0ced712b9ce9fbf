"""Tensors of another device than the current one are refused before anything is launched (on the CPU, with tensors that say that they
lie on a GPU)."""
import pytest
import torch

from paper_2602_02958_amd import binding as B


class On(torch.Tensor):
    """A host tensor that says it lies on GPU number .at."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.at


def on(t, at=0):
    t = t.as_subclass(On)
    t.at = at
    return t


def pool(units=1, **elsewhere):
    parts = dict(centroids=torch.zeros(units, 2, 4, 128, dtype=torch.bfloat16), ids=torch.zeros(units, 16, dtype=torch.uint8),
                 codes=torch.zeros(units, 16, 1, 32, dtype=torch.uint8), scales=torch.zeros(units, 16, 1, 2, dtype=torch.float16))
    return B.Encoded(*(on(t, elsewhere.get(name, 0)) for name, t in parts.items()), 8)


NAMES = ["centroids", "ids", "codes", "scales"]


@pytest.fixture(autouse=True)
def device_zero(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)

    def launched(*a):
        raise AssertionError("the call went on")
    monkeypatch.setattr(B, "_stream", launched)


@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("name", NAMES)
def test_attn_tree_refuses_a_pool_of_another_device(side, name):
    x = on(torch.zeros(1, 1, 1, 128, dtype=torch.bfloat16))
    sides = {s: pool(**({name: 1} if s == side else {})) for s in "kv"}
    with pytest.raises(ValueError, match="current device"):
        B.attn_tree(x, sides["k"], sides["v"], None, None, x, x, out=x, scratch=on(torch.zeros(0, dtype=torch.uint8)))


@pytest.mark.parametrize("side", ["cache", "into"])
@pytest.mark.parametrize("name", NAMES)
def test_copy_pages_refuses_a_pool_of_another_device(side, name):
    pools = {s: pool(**({name: 1} if s == side else {})) for s in ("cache", "into")}
    with pytest.raises(ValueError, match="current device"):
        B.copy_pages(pools["cache"], [0], [1], into=pools["into"])


def test_the_others_refuse_it_too():
    x, y = (on(torch.zeros(1, 1, 1, 128, dtype=torch.bfloat16), at) for at in (0, 1))
    i, j = (on(torch.zeros(1, 1, dtype=torch.int32), at) for at in (0, 1))
    n, m = (on(torch.zeros(1, dtype=torch.int32), at) for at in (0, 1))
    for bad in (dict(parents=j), dict(n_nodes=m), dict(depth=j)):
        with pytest.raises(ValueError, match="current device"):
            B.tree_mask(**{**dict(parents=i, n_nodes=n, mask=on(torch.zeros(1, 1, 1, dtype=torch.int32)), depth=i), **bad})
    args = dict(k_new=x, v_new=x, path=i, n_keep=n, tail_k=x, tail_v=x, tail_len=n, out_len=n)
    for name, t in args.items():
        with pytest.raises(ValueError, match="current device"):
            B.keep_nodes(**{**args, name: y if t is x else j if t is i else m})


def test_a_cache_refuses_tokens_of_another_device(monkeypatch):
    init = on(torch.zeros(2, 4, 128, dtype=torch.bfloat16))
    c = B.PagedCache(1, 1, 2, 8, 2, 4, 4, 64, 1, init, device="cpu", pre_rope=True)
    c.tail = on(c.tail)
    s = c.open()
    kv, rot = torch.zeros(2, 3, 128, dtype=torch.bfloat16), torch.zeros(1, 3, 128, dtype=torch.bfloat16)
    for a, b in ((1, 0), (0, 1)):
        with pytest.raises(ValueError, match="current device"):
            c.append(s, on(kv, a), k_rotated=on(rot, b))
    for name in ("tail", "init"):
        there = getattr(c, name)
        monkeypatch.setattr(c, name, on(there.clone(), 1))
        with pytest.raises(ValueError, match="current device"):
            c.append(s, on(kv), k_rotated=on(rot))
        monkeypatch.setattr(c, name, there)
    assert c.length(s) == 0
