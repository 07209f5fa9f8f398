"""gvote_evict's mask as gvote_vote leaves it: every word of a head's row is written, padding is zero."""
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
@pytest.mark.parametrize("lens,first", [((64, 32, 0, 33), 0), ((32,), 0), ((0, 0, 5), 0), ((131072, 96), 0), ((31, 1, 64), 100),
                                        ((0,), 7), ((40000, 8), 33)])
@pytest.mark.parametrize("kind", ["random", "all", "none", "ties"])
def test_every_word_of_the_mask_is_written(gv, lens, first, kind):
    """`first`: slots before the first request (the later requests of a batch, by a view of its boundaries)."""
    hkv, batch = 2, len(lens)
    p = gv.make_params(d_h=64, n_q_heads=2, n_kv_heads=hkv, d_k=64, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=3, seed=0)
    cu = (first + np.concatenate([[0], np.cumsum(lens)])).astype(np.int32)
    total = int(cu[-1])
    rng = np.random.default_rng(total + batch)
    acc = (rng.integers(0, 3, (hkv, total)) if kind == "ties" else rng.random((hkv, total))).astype(np.float32)
    share = {"random": 0.4, "all": 1.0, "none": 0.0, "ties": 0.5}[kind]
    keep = np.array([[int(n * share)] * hkv for n in lens], dtype=np.int32)
    geom = (batch, total, max(lens))
    mask = torch.full((hkv, gv.mask_row_words(total, batch)), -1, dtype=torch.int32).cuda()
    budget = torch.full((batch, hkv), -1, dtype=torch.int32).cuda()
    gv.gvote_evict(p, torch.from_numpy(acc).cuda(), torch.from_numpy(cu).cuda(), geom, torch.from_numpy(keep).cuda(), 2, mask, budget,
                   gv.alloc_cache_workspace(p, *geom))
    want = np.zeros((hkv, gv.mask_row_words(total, batch)), dtype=np.uint32)
    for r, n in enumerate(lens):
        for h in range(hkv):
            kept = np.flatnonzero(co.evict(acc[h, cu[r]:cu[r + 1]], int(keep[r, h]), 2, 3))
            np.bitwise_or.at(want[h], gv.mask_word_offset(int(cu[r]), r) + kept // 32, np.uint32(1) << (kept % 32).astype(np.uint32))
            assert int(budget[r, h]) == kept.size
    assert np.array_equal(mask.cpu().numpy().view(np.uint32), want)
