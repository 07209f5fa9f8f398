"""gvote_accumulate where weights lie below what 32 bits hold: they are zero, as are the weights of the keys that a query does
not see, so that what they add up to is zero and the eviction takes such keys by their slot."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def gv():
    from paper_2509_03136_b200 import build as gbuild
    gbuild.build()
    from paper_2509_03136_b200 import gvote
    gvote.load()
    return gvote


@gpu
@pytest.mark.parametrize("g,n,n_q,given_lse", [(7, 1000, 300, False), (4, 700, 40, False), (1, 5000, 1, False), (8, 400, 300, True),
                                               (3, 130, 129, False)])
def test_keys_without_weight_have_none_and_tie(gv, g, n, n_q, given_lse):
    """One early key 200 above all others (e^-200 is far below the least float): it takes everything, every other key exactly
    nothing, however many query tiles pass it."""
    p = gv.make_params(d_h=64, n_q_heads=g, n_kv_heads=1, d_k=64, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=0, seed=0)
    heavy = 0 if n_q == n - 1 else 37
    K, Q = torch.zeros(1, n, 64), torch.zeros(n_q, g, 64)
    K[0, heavy, 0], Q[:, :, 0] = 40.0, 40.0                             # 1600 / 8 = 200
    cu, cq = (torch.tensor([0, x], dtype=torch.int32).cuda() for x in (n, n_q))
    geom, acc = (1, n, n), torch.full((1, n), -1.0).cuda()
    ws = gv.alloc_cache_workspace(p, *geom, n_q, n_q)
    ws[256:].fill_(0xff)
    lse = torch.full((n_q, g), 200.0).cuda() if given_lse else None
    gv.gvote_accumulate(p, Q.bfloat16().cuda(), cq, n_q, K.bfloat16().cuda(), cu, geom, acc, ws, lse=lse)
    got = acc[0].cpu().numpy()
    assert np.array_equal(np.flatnonzero(got), [heavy])
    assert abs(got[heavy] - n_q * g) <= (200 * 2.0 ** -21 + 2.0 ** -20) * n_q * g
    keep, mask = torch.tensor([[20]], dtype=torch.int32).cuda(), torch.zeros(1, gv.mask_row_words(n, 1), dtype=torch.int32).cuda()
    gv.gvote_evict(p, acc, cu, geom, keep, 0, mask, torch.zeros(1, 1, dtype=torch.int32).cuda(), ws)
    assert gv.gvote_poll_status(ws) == 0
    kept = np.flatnonzero(gv.unpack_mask(mask[0].cpu().numpy(), 0, n))
    assert np.array_equal(kept, np.flatnonzero(co.evict(np.eye(1, n, heavy)[0], 20, 0, 0)))


@gpu
def test_a_query_that_sees_no_key_adds_nothing(gv):
    """Five rows, eight query tokens: the first three see none."""
    p = gv.make_params(d_h=64, n_q_heads=4, n_kv_heads=2, d_k=32, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=0, seed=0)
    rng = np.random.default_rng(3)
    K, Q = torch.zeros(2, 5, 32), torch.zeros(8, 4, 32)
    K[:, 0, 0], Q[:, :, 0] = 100.0, 100.0                               # the first key takes it all
    cu, cq = (torch.tensor([0, x], dtype=torch.int32).cuda() for x in (5, 8))
    acc = torch.full((2, 5), -1.0).cuda()
    ws = gv.alloc_cache_workspace(p, 1, 5, 5, 8, 8)
    ws[256:].fill_(0xff)
    gv.gvote_accumulate(p, Q.bfloat16().cuda(), cq, 8, K.bfloat16().cuda(), cu, (1, 5, 5), acc, ws)
    got = acc.double().cpu().numpy()
    assert (got[:, 1:] == 0).all()
    # 10 weights of 1; the logits are 1e4 / sqrt(32), and the log-sum-exp enters the exponent in 32 bits
    assert (np.abs(got[:, 0] - 10) <= 10 * (1e4 / 32 ** 0.5 * 2.0 ** -21 + 2.0 ** -20)).all()
