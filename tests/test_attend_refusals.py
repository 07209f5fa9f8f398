"""What the entry points of the paged cache and of the attention over bf16 rows refuse, on the host, before anything is enqueued.
CPU only: the device pointers are numbers that nothing reads."""
import ctypes
import os
import re

import pytest
import torch

from paper_2509_03136_b200 import build as gbuild

A = 1 << 20            # a 16-byte aligned "device pointer"
INVALID, UNALIGNED, SMALL, SHAPE = -1, -2, -3, -4
OPS = ["tables", "write", "pages", "slabs"]


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


def _pages(gv, **kw):
    base = dict(K=A, V=2 * A, tables=3 * A, kv_len=4 * A, free_pages=5 * A, n_free=6 * A, row_stride=64, page_stride=64 * 16,
                n_pages=100, page_rows=16, max_pages=50, batch=2)
    base.update(kw)
    return gv.GVotePages(*[base[f[0]] for f in gv.GVotePages._fields_])


def _call(gv, op, p=None, pages=None, ws_bytes=1 << 40, **kw):
    lib, b = gv.load(), ctypes.byref
    p, g = p or _p(gv), b(pages or _pages(gv))
    d = dict(K=21 * A, V=22 * A, tok=64, head=64 * 512, cu=24 * A, kv=25 * A, batch=2, total=512, max_N=300, keep=26 * A,
             cu_new=30 * A, total_new=8, max_new=4, mask=31 * A, slots=32 * A, Q=33 * A, q_tok=512, q_head=64, cu_q=34 * A, total_q=8,
             max_q=4, out=35 * A, o_tok=512, o_head=64, lse=36 * A, ws=38 * A)
    d.update(kw)
    f = lambda names: [d[n] for n in names.split()]
    tail = [d["ws"], ws_bytes, 0]
    if op == "tables":
        return lib.gvote_page_tables(b(p), g, *f("keep cu_new total_new max_new mask slots"), *tail)
    if op == "write":
        return lib.gvote_page_write(b(p), *f("K V tok head slots total_new"), g, *tail)
    if op == "pages":
        return lib.gvote_page_attend(b(p), *f("Q q_tok q_head cu_q total_q max_q"), g, *f("out o_tok o_head lse"), *tail)
    return lib.gvote_attend(b(p), *f("Q q_tok q_head cu_q total_q max_q K V tok head cu kv batch total max_N out o_tok o_head lse"), *tail)


@pytest.mark.parametrize("op", OPS)
def test_shapes_and_workspace(gv, op):
    n0 = gv.gvote_launch_count()
    assert _call(gv, op, p=_p(gv, d_k=72)) == SHAPE                    # not a multiple of 16
    assert _call(gv, op, p=_p(gv, d_k=272)) == SHAPE                   # above 256
    assert _call(gv, op, p=_p(gv, n_q_heads=258)) == SHAPE             # 129 query heads per KV head
    assert _call(gv, op, p=_p(gv, n_q_heads=1025, n_kv_heads=1025)) == SHAPE
    assert _call(gv, op, p=_p(gv, n_q_heads=7)) == INVALID
    assert _call(gv, op, ws_bytes=16) == SMALL
    assert _call(gv, op, ws=None) == INVALID
    assert _call(gv, op, ws=A + 8) == UNALIGNED
    assert gv.gvote_launch_count() == n0


@pytest.mark.parametrize("op", ["tables", "write", "pages"])
@pytest.mark.parametrize("field,value,status", [
    ("K", 0, INVALID), ("V", 0, INVALID), ("tables", 0, INVALID), ("kv_len", 0, INVALID), ("K", A + 2, UNALIGNED),
    ("tables", A + 4, UNALIGNED), ("n_pages", 0, INVALID), ("max_pages", 0, INVALID), ("batch", 0, INVALID),
    ("batch", 65536, SHAPE), ("page_rows", 8, SHAPE), ("page_rows", 48, SHAPE), ("page_rows", 2048, SHAPE),
    ("n_pages", 1 << 27, SHAPE), ("max_pages", (1 << 22) + 1, SHAPE), ("row_stride", 56, UNALIGNED), ("row_stride", 68, UNALIGNED),
    ("page_stride", 1028, UNALIGNED), ("page_stride", 1 << 38, SHAPE)])
def test_page_block(gv, op, field, value, status):
    assert _call(gv, op, pages=_pages(gv, **{field: value})) == status


@pytest.mark.parametrize("op,changes,status", [
    ("tables", dict(max_new=9), INVALID), ("tables", dict(total_new=-1), INVALID), ("tables", dict(cu_new=None), INVALID),
    ("tables", dict(cu_new=None, total_new=0, max_new=0), INVALID), ("tables", dict(total_new=(1 << 30) + 1), SHAPE),
    ("tables", dict(keep=A + 4), UNALIGNED), ("tables", dict(mask=A + 4), UNALIGNED), ("tables", dict(slots=A + 4), UNALIGNED),
    ("write", dict(K=None), INVALID), ("write", dict(V=None), INVALID), ("write", dict(slots=None), INVALID),
    ("write", dict(total_new=-1), INVALID), ("write", dict(tok=60), UNALIGNED), ("write", dict(head=60), UNALIGNED),
    ("pages", dict(Q=None), INVALID), ("pages", dict(out=None), INVALID), ("pages", dict(cu_q=None), INVALID),
    ("pages", dict(max_q=0), INVALID), ("pages", dict(max_q=9), INVALID), ("pages", dict(q_head=60), UNALIGNED),
    ("pages", dict(q_tok=508), UNALIGNED), ("pages", dict(o_tok=4), UNALIGNED), ("pages", dict(o_head=32), UNALIGNED),
    ("pages", dict(lse=A + 4), UNALIGNED), ("pages", dict(total_q=(1 << 30) + 1), SHAPE),
    ("slabs", dict(Q=None), INVALID), ("slabs", dict(K=None), INVALID), ("slabs", dict(V=None), INVALID), ("slabs", dict(cu=None), INVALID),
    ("slabs", dict(out=None), INVALID), ("slabs", dict(batch=0), INVALID), ("slabs", dict(max_N=513), INVALID),
    ("slabs", dict(total=(1 << 30) + 1), SHAPE), ("slabs", dict(tok=60), UNALIGNED), ("slabs", dict(head=60), UNALIGNED),
    ("slabs", dict(kv=A + 4), UNALIGNED), ("slabs", dict(max_q=0), INVALID), ("slabs", dict(batch=65536), SHAPE)])
def test_arguments(gv, op, changes, status):
    assert _call(gv, op, **changes) == status


def test_stacks_are_needed_for_tables_only(gv):
    for field in ("free_pages", "n_free"):
        assert _call(gv, "tables", pages=_pages(gv, **{field: 0})) == INVALID


@pytest.mark.parametrize("op", ["pages", "slabs"])
def test_wide_heads_take_a_few_tokens(gv, op):
    wide = dict(p=_p(gv, d_k=144), pages=_pages(gv, row_stride=144, page_stride=144 * 16), tok=144, head=144 * 512, q_head=144,
                q_tok=8 * 144, o_head=144, o_tok=8 * 144)
    assert _call(gv, op, **wide, total_q=64, max_q=33) == SHAPE
    assert _call(gv, op, **wide, total_q=64, max_q=32, ws_bytes=16) == SMALL


def test_workspace_serves_smaller_calls(gv):
    size = lambda p, *s: gv.load().gvote_attend_workspace_bytes(ctypes.byref(p), *s)
    for p in (_p(gv), _p(gv, n_q_heads=28, n_kv_heads=4, d_k=128), _p(gv, n_q_heads=128, n_kv_heads=1), _p(gv, d_k=256)):
        last = 0
        for n in (0, 1, 2, 5, 8, 17, 32) + (() if p.d_k > 128 else (33, 64, 100, 1000, 20000)):
            now = size(p, 3, 3 * n, n)
            assert now >= last > -1 and now > 256
            assert all(size(p, b, b * n, n) <= now for b in (1, 2))
            last = now
    for bad in ((0, 1, 1), (1, 1, 2), (1, -1, 0), (65536, 1, 1)):
        assert size(_p(gv), *bad) == 0
    with pytest.raises(gv.GVoteError):
        gv.alloc_attend_workspace(_p(gv), 1, 1, 2)


def test_page_struct_matches_header(gv):
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gvote.h")).read()
    body = re.search(r"typedef struct \{([^}]*)\} gvote_pages;", header, re.S).group(1)
    fields = re.findall(r"(\w+);", re.sub(r"/\*.*?\*/", "", body, flags=re.S))
    assert fields == [f[0] for f in gv.GVotePages._fields_] and ctypes.sizeof(gv.GVotePages) == 80
    assert f"#define GVOTE_ATTEND_FEW_Q {gv.ATTEND_FEW_Q}\n" in header


def test_python_face_refuses_tensors_of_the_wrong_kind(gv):
    z = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype)
    bf = lambda *s: z(*s, dtype=torch.bfloat16)
    args = lambda **kw: {**dict(K=bf(9, 16, 64), V=bf(9, 16, 64), tables=z(1, 2, 3), kv_len=z(1, 2), free=z(9), n_free=z(1)), **kw}
    with pytest.raises(TypeError, match="CUDA"):
        gv.PageCache(**args())
    with pytest.raises(TypeError, match="bfloat16"):
        gv.PageCache(**args(K=z(9, 16, 64), V=z(9, 16, 64)))
    with pytest.raises(ValueError, match="strides"):
        gv.PageCache(**args(K=bf(16, 9, 64).transpose(0, 1)))
    with pytest.raises((TypeError, ValueError)):                       # (the first tensor is refused for its device already)
        gv.PageCache(**args(kv_len=z(2, 1)))
