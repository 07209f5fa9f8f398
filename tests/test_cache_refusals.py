"""What the entry points of the 8-bit cache and the eviction refuse, on the host, before anything is enqueued.
CPU only: the device pointers are numbers that nothing reads."""
import ctypes

import pytest
import torch

from paper_2509_03136_b200 import build as gbuild

A = 1 << 20            # a 16-byte aligned "device pointer"


@pytest.fixture(scope="module")
def gv():
    gbuild.build()
    from paper_2509_03136_b200 import gvote
    gvote.load()
    return gvote


def _p(gv, **kw):
    base = dict(d_h=64, n_q_heads=8, n_kv_heads=2, d_k=64, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=4, seed=0)
    base.update(kw)
    return gv.make_params(**base)


def _cache(gv, **kw):
    base = dict(K=A, V=2 * A, k_scale=3 * A, v_scale=4 * A, cu_seqlens=5 * A, kv_len=6 * A, tok_stride=64,
                head_stride=64 * 512, total_tokens=512, max_N=512, batch=1, reserved=0)
    base.update(kw)
    return gv.GVoteCache8(*[base[f[0]] for f in gv.GVoteCache8._fields_])


def _call(gv, op, p=None, cache=None, other=None, ws_bytes=1 << 40, **kw):
    lib, b = gv.load(), ctypes.byref
    p, c, o = p or _p(gv), cache or _cache(gv), other or _cache(gv, K=11 * A, V=12 * A, k_scale=13 * A, v_scale=14 * A, kv_len=16 * A)
    d = dict(K=21 * A, V=22 * A, tok=64, head=64 * 512, mask=23 * A, cu=24 * A, kv=25 * A, batch=1, total=512, max_N=512,
             acc=26 * A, acc_out=27 * A, pos=28 * A, pos_out=29 * A, cu_new=30 * A, total_new=4, max_new=4, kv_out=31 * A,
             pos_new=32 * A, Q=33 * A, q_tok=512, q_head=64, total_q=4, max_q=4, out=34 * A, o_tok=512, o_head=64,
             lse=35 * A, keep=36 * A, n_recent=1, budget=37 * A, ws=38 * A)
    d.update(kw)
    g = lambda names: [d[n] for n in names.split()]
    tail = [d["ws"], ws_bytes, 0]
    if op == "store":
        return lib.gvote_store8(b(p), *g("K V tok head mask cu kv batch total max_N"), b(c), *g("acc acc_out pos pos_out"), *tail)
    if op == "prune":
        return lib.gvote_prune8(b(p), b(c), d["mask"], b(o), *g("acc acc_out pos pos_out"), *tail)
    if op == "append":
        return lib.gvote_append8(b(p), *g("K V tok head cu_new total_new max_new"), b(c), *g("kv_out acc pos pos_new"), *tail)
    if op == "attend":
        return lib.gvote_attend8(b(p), *g("Q q_tok q_head cu_new total_q max_q"), b(c), *g("out o_tok o_head lse acc acc_out"), *tail)
    if op == "accumulate":
        return lib.gvote_accumulate(b(p), *g("Q q_tok q_head cu_new total_q max_q K tok head cu kv batch total max_N lse acc acc_out"), *tail)
    return lib.gvote_evict(b(p), *g("acc cu kv batch total max_N keep n_recent mask budget"), *tail)


INVALID, UNALIGNED, SMALL, SHAPE = -1, -2, -3, -4
OPS = ["store", "prune", "append", "attend", "accumulate", "evict"]


@pytest.mark.parametrize("op", OPS)
def test_shapes_and_workspace(gv, op):
    n0 = gv.gvote_launch_count()
    assert _call(gv, op, p=_p(gv, d_k=72)) == SHAPE                    # not a multiple of 16
    assert _call(gv, op, p=_p(gv, d_k=272)) == SHAPE                   # above 256
    assert _call(gv, op, p=_p(gv, n_q_heads=258)) == SHAPE             # 129 query heads per KV head
    assert _call(gv, op, p=_p(gv, n_q_heads=7)) == INVALID
    assert _call(gv, op, ws_bytes=16) == SMALL
    assert _call(gv, op, ws=None) == INVALID
    assert _call(gv, op, ws=A + 8) == UNALIGNED
    if op in ("prune", "append", "attend"):
        assert _call(gv, op, cache=_cache(gv, batch=0)) == INVALID
        assert _call(gv, op, cache=_cache(gv, max_N=513)) == INVALID
        assert _call(gv, op, cache=_cache(gv, batch=70000)) == SHAPE
    else:
        assert _call(gv, op, batch=0) == INVALID
        assert _call(gv, op, max_N=513) == INVALID
        assert _call(gv, op, batch=70000) == SHAPE
        assert _call(gv, op, total=(1 << 30) + 1) == SHAPE
    assert gv.gvote_launch_count() == n0


@pytest.mark.parametrize("op", ["store", "prune", "append", "attend"])
@pytest.mark.parametrize("field,value,status", [("K", 0, INVALID), ("V", 0, INVALID), ("k_scale", 0, INVALID),
                                                ("v_scale", 0, INVALID), ("cu_seqlens", 0, INVALID), ("kv_len", 0, INVALID),
                                                ("K", A + 1, UNALIGNED), ("tok_stride", 48, UNALIGNED),
                                                ("tok_stride", 72, UNALIGNED), ("head_stride", 8, UNALIGNED)])
def test_cache_block(gv, op, field, value, status):
    assert _call(gv, op, cache=_cache(gv, **{field: value})) == status


@pytest.mark.parametrize("op,changes,status", [
    ("store", dict(K=None), INVALID), ("store", dict(V=None), INVALID), ("store", dict(cu=None), INVALID),
    ("store", dict(acc_out=None), INVALID), ("store", dict(acc=None), INVALID), ("store", dict(pos_out=None), INVALID),
    ("store", dict(acc_out=26 * A), INVALID), ("store", dict(pos_out=28 * A), INVALID), ("store", dict(kv=6 * A), INVALID),
    ("store", dict(tok=56), UNALIGNED), ("store", dict(tok=68), UNALIGNED), ("store", dict(mask=A + 4), UNALIGNED),
    ("store", dict(batch=2), INVALID),
    ("prune", dict(acc_out=None), INVALID), ("prune", dict(pos_out=None), INVALID), ("prune", dict(acc_out=26 * A), INVALID),
    ("append", dict(K=None), INVALID), ("append", dict(cu_new=None), INVALID), ("append", dict(kv_out=None), INVALID),
    ("append", dict(max_new=5), INVALID), ("append", dict(total_new=-1), INVALID), ("append", dict(pos_new=None), INVALID),
    ("append", dict(pos=None), INVALID), ("append", dict(tok=60), UNALIGNED),
    ("attend", dict(Q=None), INVALID), ("attend", dict(out=None), INVALID), ("attend", dict(acc_out=None), INVALID),
    ("attend", dict(max_q=0), INVALID), ("attend", dict(max_q=5), INVALID), ("attend", dict(total_q=33, max_q=33), SHAPE),
    ("attend", dict(q_head=60), UNALIGNED), ("attend", dict(o_tok=4), UNALIGNED), ("attend", dict(lse=A + 4), UNALIGNED),
    ("accumulate", dict(Q=None), INVALID), ("accumulate", dict(K=None), INVALID), ("accumulate", dict(acc_out=None), INVALID),
    ("accumulate", dict(max_q=0), INVALID), ("accumulate", dict(q_head=60), UNALIGNED), ("accumulate", dict(tok=60), UNALIGNED),
    ("evict", dict(acc=None), INVALID), ("evict", dict(keep=None), INVALID), ("evict", dict(mask=None), INVALID),
    ("evict", dict(budget=None), INVALID), ("evict", dict(n_recent=-1), INVALID),
])
def test_arguments(gv, op, changes, status):
    assert _call(gv, op, **changes) == status


def test_prune_refuses_to_work_in_place(gv):
    for field in ("K", "V", "k_scale", "v_scale", "kv_len"):
        o = _cache(gv, **{**dict(K=11 * A, V=12 * A, k_scale=13 * A, v_scale=14 * A, kv_len=16 * A),
                          field: getattr(_cache(gv), field)})
        assert _call(gv, "prune", other=o) == INVALID, field


def test_workspace_size(gv):
    p = _p(gv)
    a = gv.load().gvote_cache_workspace_bytes(ctypes.byref(p), 1, 512, 512, 0, 0)
    b = gv.load().gvote_cache_workspace_bytes(ctypes.byref(p), 1, 512, 512, 8, 8)
    assert 256 < a < b
    for bad in ((0, 512, 512, 0, 0), (1, 512, 513, 0, 0), (1, 512, 512, 1, 2), (1, 512, 512, -1, 0)):
        assert gv.load().gvote_cache_workspace_bytes(ctypes.byref(p), *bad) == 0
    with pytest.raises(gv.GVoteError):
        gv.alloc_cache_workspace(p, 1, 512, 513)


def test_cache_struct_matches_header(gv):
    import os, re
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gvote.h")).read()
    body = re.search(r"typedef struct \{([^}]*)\} gvote_cache8;", header, re.S).group(1)
    fields = re.findall(r"(\w+);", re.sub(r"/\*.*?\*/", "", body, flags=re.S))
    assert fields == [f[0] for f in gv.GVoteCache8._fields_] and ctypes.sizeof(gv.GVoteCache8) == 88


def test_python_face_refuses_tensors_of_the_wrong_kind(gv):
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)
    args = lambda **kw: {**dict(K=z(2, 64, 64, dtype=torch.uint8), V=z(2, 64, 64, dtype=torch.uint8), k_scale=z(2, 2),
                                v_scale=z(2, 2), cu_seqlens=z(2, dtype=torch.int32), kv_len=z(1, 2, dtype=torch.int32),
                                geom=(1, 64, 64)), **kw}
    with pytest.raises(TypeError, match="CUDA"):
        gv.Cache8(**args())
    with pytest.raises(TypeError, match="uint8"):
        gv.Cache8(**args(K=z(2, 64, 64)))
    with pytest.raises(ValueError, match="strides"):
        gv.Cache8(**args(K=z(64, 2, 64, dtype=torch.uint8).transpose(0, 1)))
    with pytest.raises(ValueError, match="shape"):
        gv.Cache8(**args(K=z(2, 63, 64, dtype=torch.uint8), V=z(2, 63, 64, dtype=torch.uint8)))
