"""gvote_prune8 and gvote_store8 work out of place, in no order: what they read and what they write must not share a byte, and the
entry points refuse it, on the host.  A workspace that is too small ends the calls that pass that check, so the
device pointers are numbers that nothing reads.  CPU only."""
import ctypes

import pytest

A = 1 << 30
INVALID, SMALL = -1, -3
H, T, D = 2, 512, 64


@pytest.fixture(scope="module")
def gv():
    from paper_2509_03136_b200 import build as gbuild
    gbuild.build()
    from paper_2509_03136_b200 import gvote
    gvote.load()
    return gvote


def cache(gv, **kw):
    base = dict(K=A, V=2 * A, k_scale=3 * A, v_scale=4 * A, cu_seqlens=5 * A, kv_len=6 * A, tok_stride=D, head_stride=D * T,
                total_tokens=T, max_N=T, batch=1, reserved=0)
    base.update(kw)
    return gv.GVoteCache8(*[base[f[0]] for f in gv.GVoteCache8._fields_])


def other(gv, **kw):
    return cache(gv, **{**dict(K=11 * A, V=12 * A, k_scale=13 * A, v_scale=14 * A, kv_len=16 * A), **kw})


def params(gv, heads=H):
    return gv.make_params(d_h=64, n_q_heads=4 * heads, n_kv_heads=heads, d_k=D, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=4, seed=0)


def prune(gv, src, dst, acc=21 * A, acc_out=22 * A, pos=23 * A, pos_out=24 * A, heads=H):
    p = params(gv, heads)
    return gv.load().gvote_prune8(ctypes.byref(p), ctypes.byref(src), None, ctypes.byref(dst), acc, acc_out, pos, pos_out, 25 * A, 256, 0)


def store(gv, dst, K=31 * A, V=32 * A, tok=D, head=D * T, kv=33 * A, acc=21 * A, acc_out=22 * A):
    p = params(gv)
    return gv.load().gvote_store8(ctypes.byref(p), K, V, tok, head, None, 5 * A, kv, 1, T, T, ctypes.byref(dst), acc, acc_out, None, None,
                                  25 * A, 256, 0)


LAST = (H - 1) * D * T + (T - 1) * D          # of the codes: the last row's offset


def test_buffers_of_their_own_pass(gv):
    assert prune(gv, cache(gv), other(gv)) == SMALL and store(gv, other(gv)) == SMALL


@pytest.mark.parametrize("off,status", [(0, INVALID), (16, INVALID), (D, INVALID), (-D * (T - 1), INVALID), (LAST, INVALID), (-LAST, INVALID),
                                        (LAST + D, SMALL), (-LAST - D, SMALL)])
@pytest.mark.parametrize("read,write", [("K", "K"), ("V", "V"), ("K", "V"), ("V", "K")])
def test_codes_that_share_bytes(gv, off, status, read, write):
    src = cache(gv)
    assert prune(gv, src, other(gv, **{write: getattr(src, read) + off})) == status


@pytest.mark.parametrize("field,size", [("k_scale", 4 * H * (T // 64 + 1)), ("v_scale", 4 * H * (T // 64 + 1)), ("kv_len", 16)])
def test_small_arrays_that_share_bytes(gv, field, size):
    src = cache(gv)
    whole = (size + 15) // 16 * 16
    for off in (0, 16, -16) if size > 16 else (0,):
        assert prune(gv, src, other(gv, **{field: getattr(src, field) + off})) == INVALID
    for off in (whole, -whole):
        assert prune(gv, src, other(gv, **{field: getattr(src, field) + off})) == SMALL


def test_side_arrays_that_share_bytes(gv):
    n = 4 * H * T
    for call, c in ((lambda **kw: prune(gv, cache(gv), other(gv), **kw), None), (lambda **kw: store(gv, other(gv), **kw), None)):
        for off in (0, 16, -16, n - 16):
            assert call(acc_out=21 * A + off) == INVALID
        assert call(acc_out=21 * A + n) == SMALL
    assert prune(gv, cache(gv), other(gv), pos_out=23 * A + 64) == INVALID


@pytest.mark.parametrize("other_row,status", [(D, SMALL), (D + 16, SMALL), (D - 16, INVALID), (2 * D + 16, INVALID), (3 * D, INVALID), (3 * D + 32, SMALL)])
def test_rows_that_lie_between_each_other(gv, other_row, status):
    """Two caches as windows of one buffer of wider rows share its extent, but no byte, as long as the windows do not meet."""
    wide = dict(tok_stride=2 * D + 32, head_stride=(2 * D + 32) * T)
    src = cache(gv, **wide)
    assert prune(gv, src, other(gv, K=src.K + other_row, **wide)) == status


def test_heads_that_lie_between_each_other(gv):
    far = dict(head_stride=2 * D * T)
    assert prune(gv, cache(gv, **far), other(gv, K=A + D * T, **far)) == SMALL
    assert prune(gv, cache(gv, **far), other(gv, K=A + D * T - D, **far)) == INVALID
    assert prune(gv, cache(gv, **far), other(gv, K=A + D * T, **far), heads=1) == SMALL
    # strides that differ: nothing is worked out, a common extent is refused
    assert prune(gv, cache(gv, **far), other(gv, K=A + D * T, head_stride=D * T)) == INVALID


def test_store_refuses_rows_that_lie_in_the_cache(gv):
    c = other(gv)
    for K in (c.K, c.K + D, c.V, c.K - 2 * LAST):
        assert store(gv, c, K=K) == INVALID and store(gv, c, V=K) == INVALID
    assert store(gv, c, K=c.K + LAST + D) == SMALL and store(gv, c, kv=16 * A) == INVALID


def test_against_counting_the_bytes(gv):
    import random
    rng = random.Random(3)
    seen = set()
    for _ in range(3000):
        heads, t1, t2 = rng.randint(1, 4), rng.randint(1, 6), rng.randint(1, 6)
        tok = 16 * rng.randint(4, 12)
        head = rng.choice([tok * max(t1, t2), 16 * rng.randint(1, 60), tok * 16])
        lie = dict(tok_stride=tok, head_stride=head, max_N=1)
        src = cache(gv, total_tokens=t1, **lie)
        dst = other(gv, total_tokens=t2, K=A + 16 * rng.randint(-80, 80), **lie)
        cells = [{base + h * head + t * tok + c for h in range(heads) for t in range(n) for c in range(0, D, 16)}
                 for base, n in ((src.K, t1), (dst.K, t2))]
        want = INVALID if cells[0] & cells[1] else SMALL
        seen.add(want)
        assert prune(gv, src, dst, heads=heads) == want, (heads, t1, t2, tok, head, dst.K - A)
    assert len(seen) == 2
