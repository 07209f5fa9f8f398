"""A cache on another device than the tensors of the call is refused by every entry point that takes one: its pointers would
be read on a device that cannot.  CPU only: the checks look at a tensor's type, shape and device, and no launch is reached."""
from types import SimpleNamespace

import pytest
import torch

HERE, THERE = torch.device("cuda", 0), torch.device("cuda", 1)


class FakeTensor:
    """What the checks ask of a tensor."""

    def __init__(self, shape, dtype, device):
        self.t, self.dtype, self.device, self.is_cuda = torch.empty(shape, dtype=dtype, device="meta"), dtype, device, True
        self.shape = self.t.shape

    def stride(self, *i):
        return self.t.stride(*i)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def gv(monkeypatch):
    from paper_2509_03136_b200 import build as gbuild
    gbuild.build()
    from paper_2509_03136_b200 import gvote
    gvote.load()

    def no_launch(*a, **kw):
        raise AssertionError("the call reached its launch")
    monkeypatch.setattr(gvote, "_launch", no_launch)
    return gvote


def calls(gv, dev, cache, other):
    p = gv.make_params(d_h=64, n_q_heads=8, n_kv_heads=2, d_k=64, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=4, seed=0)
    t = lambda dtype, *s: FakeTensor(s, dtype, dev)
    bf, i32 = torch.bfloat16, torch.int32
    rows, geom = t(bf, 2, 100, 64), (1, 100, 100)
    return {
        "store": lambda: gv.gvote_store8(p, rows, rows, t(i32, 2), geom, cache, None),
        "prune": lambda: gv.gvote_prune8(p, cache, None, other, None),
        "append": lambda: gv.gvote_append8(p, rows, rows, t(i32, 2), 100, cache, t(i32, 1, 2), None),
        "attend": lambda: gv.gvote_attend8(p, t(bf, 1, 8, 64), t(i32, 2), 1, cache, t(bf, 1, 8, 64), None),
    }


def cache(gv, dev):
    return SimpleNamespace(shape=(2, 64), device=dev, geom=(1, 100, 100), args=gv.GVoteCache8(), kv_len=None)


@pytest.mark.parametrize("op", ["store", "prune", "append", "attend"])
def test_cache_on_another_device(gv, op):
    with pytest.raises(ValueError, match="is on cuda"):
        calls(gv, HERE, cache(gv, THERE if op != "prune" else HERE), cache(gv, THERE))[op]()
    with pytest.raises(AssertionError, match="reached"):            # the same call on one device passes the checks
        calls(gv, HERE, cache(gv, HERE), cache(gv, HERE))[op]()
