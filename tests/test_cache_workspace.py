"""gvote_cache_workspace_bytes against what the entry points demand, on the host.  A key stride that no tensor map takes
ends every call that passes the workspace check before anything is enqueued, so the device pointers are numbers
that nothing reads.  CPU only."""
import ctypes
import random

import pytest

A = 1 << 20
SMALL, SHAPE = -3, -4
NO_MAP = 1 << 45            # elements between keys: beyond what a tensor map's strides hold


@pytest.fixture(scope="module")
def gv():
    from paper_2509_03136_b200 import build as gbuild
    gbuild.build()
    from paper_2509_03136_b200 import gvote
    gvote.load()
    return gvote


def params(gv, hkv, g, d):
    return gv.make_params(d_h=64, n_q_heads=hkv * g, n_kv_heads=hkv, d_k=d, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=4, seed=0)


def size(gv, p, batch, total, max_n, total_q, max_q):
    return gv.load().gvote_cache_workspace_bytes(ctypes.byref(p), batch, total, max_n, total_q, max_q)


def accumulate(gv, p, ws_bytes, batch, total, max_n, total_q, max_q):
    return gv.load().gvote_accumulate(ctypes.byref(p), A, p.n_q_heads * p.d_k, p.d_k, 2 * A, total_q, max_q, 3 * A, NO_MAP, p.d_k,
                                      4 * A, None, batch, total, max_n, None, None, 5 * A, 6 * A, ws_bytes, 0)


def attend(gv, p, ws_bytes, batch, total, max_n, total_q, max_q, acc_out=11 * A):
    c = gv.GVoteCache8(A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, NO_MAP, p.d_k, total, max_n, batch, 0)
    return gv.load().gvote_attend8(ctypes.byref(p), 7 * A, p.n_q_heads * p.d_k, p.d_k, 8 * A, total_q, max_q, ctypes.byref(c), 9 * A,
                                   p.n_q_heads * p.d_k, p.d_k, None, None, acc_out, 10 * A, ws_bytes, 0)


def test_the_calls_here_end_before_a_launch(gv):
    p = params(gv, 2, 4, 64)
    n0 = gv.gvote_launch_count()
    for call in (accumulate, attend):
        assert call(gv, p, 1 << 40, 1, 500, 500, 8, 8) == SHAPE and call(gv, p, 256, 1, 500, 500, 8, 8) == SMALL
    assert gv.gvote_launch_count() == n0


@pytest.mark.parametrize("hkv,g,d,batch,total,max_n,total_q,max_q", [
    (8, 4, 16, 1, 20000, 1000, 20000, 1),          # one request behind others, by a view of the boundaries
    (8, 4, 128, 3, 60000, 1000, 60000, 40), (1, 1, 16, 1, 12062, 12062, 1708, 1708), (1, 1, 16, 1, 10880, 10880, 1792, 1792),
    (4, 7, 128, 1, 131072, 131072, 32, 32), (8, 4, 128, 1, 32768, 32768, 32768, 32768), (1, 128, 64, 1, 90, 90, 70, 70)])
def test_the_size_suffices_for_its_own_call(gv, hkv, g, d, batch, total, max_n, total_q, max_q):
    p = params(gv, hkv, g, d)
    n = size(gv, p, batch, total, max_n, total_q, max_q)
    assert n > 256 and accumulate(gv, p, n, batch, total, max_n, total_q, max_q) == SHAPE


def test_the_size_suffices_for_every_smaller_call(gv):
    rng = random.Random(7)
    pick = lambda top: max(1, int(top ** rng.random()))
    n0 = gv.gvote_launch_count()
    for _ in range(6000):
        hkv, g = rng.choice([(1, 1), (1, 3), (2, 2), (1, 128), (8, 4), (4, 7), (3, 5), (32, 1), (2, 40)])
        p = params(gv, hkv, g, rng.choice([16, 64, 256]))
        batch = rng.choice([1, 1, 2, 5, 40])
        total, total_q = pick(200000), pick(60000)
        max_n, max_q = rng.choice([pick(total), total]), rng.choice([pick(total_q), total_q, pick(min(total_q, 64))])
        n = size(gv, p, batch, total, max_n, total_q, max_q)
        assert n > 256
        for k in range(4):
            b, t, q = (batch, total, total_q) if k == 0 else (rng.randint(1, batch), pick(total), pick(total_q))
            mn, mq = (max_n, max_q) if k == 0 else (min(max_n, pick(t)), min(max_q, pick(q)))
            assert accumulate(gv, p, n, b, t, mn, q, mq) == SHAPE, (hkv, g, p.d_k, (batch, total, max_n, total_q, max_q), (b, t, mn, q, mq))
            if mq <= gv.ATTEND8_MAX_Q:
                assert attend(gv, p, n, b, t, mn, q, mq) == SHAPE, (hkv, g, p.d_k, (batch, total, max_n, total_q, max_q), (b, t, mn, q, mq))
    assert gv.gvote_launch_count() == n0


@pytest.mark.parametrize("hkv,g,d,batch,total,total_q,max_q", [(8, 4, 128, 1, 1 << 20, 32, 32), (2, 4, 64, 3, 5000, 3, 1), (1, 1, 16, 1, 64, 1, 1),
                                                              (4, 7, 256, 2, 131072, 40, 20)])
def test_attention_without_weights_needs_no_room_for_logits(gv, hkv, g, d, batch, total, total_q, max_q):
    p = params(gv, hkv, g, d)
    n = size(gv, p, batch, total, total, total_q, max_q) - 4 * hkv * g * max_q * total
    assert attend(gv, p, n, batch, total, total, total_q, max_q, acc_out=None) == SHAPE
    assert attend(gv, p, 4 * hkv * g * max_q * total, batch, total, total, total_q, max_q) == SMALL
    assert attend(gv, p, 256, batch, total, total, total_q, max_q, acc_out=None) == SMALL
