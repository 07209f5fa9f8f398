"""gvote_prune8 at the ends of the range: a bf16 value next to the largest is stored as 2^128 = code 256 times scale 2^120, which
no 32-bit float holds, and is a number all the same; zeros of a block with a large scale move to one with the least."""
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


def read(c, codes, scale, n):
    return codes[0, :n].view(torch.float8_e4m3fn).double().cpu().numpy(), scale[0, :(n + 63) // 64].double().cpu().numpy()


@gpu
@pytest.mark.parametrize("keep", ["all", "odd", "late"])
def test_values_beyond_the_largest_float_and_zeros_across_all_scales(gv, keep):
    n, d = 448, 32
    x = np.zeros((n, d), dtype=np.float32)
    big = 3.3895e38
    x[0:64, 3] = 2.0 ** 100                          # beside the largest: moves by 2^20
    x[5, 1], x[6, 2], x[7, 0] = big, -big, np.inf
    x[64:128, 0] = 2.0 ** -120                       # tiny, kept into a block with the largest ones
    x[130, 4] = big                                  # a block that is zero but for one row, which is not kept
    x[192:256, 7] = np.linspace(-448, 448, 64) * 2.0 ** -126
    x[256:320] = 2.0 ** -133
    x[320, 0], x[321, 0] = 1.0, np.nan
    flags = {"all": np.ones(n, bool), "odd": np.arange(n) % 2 == 1, "late": np.arange(n) >= 70}[keep].copy()
    flags[130] = False
    K = torch.from_numpy(x).bfloat16()[None]
    V = torch.flip(K, dims=[2]).contiguous()
    p = gv.make_params(d_h=64, n_q_heads=1, n_kv_heads=1, d_k=d, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=0, seed=0)
    c, out = (gv.alloc_cache8(p, [0, n]) for _ in range(2))
    ws = gv.alloc_cache_workspace(p, *c.geom)
    gv.gvote_store8(p, K.cuda(), V.cuda(), c.cu_seqlens, c.geom, c, ws)
    words = np.zeros(gv.mask_row_words(n, 1), dtype=np.uint32)
    idx = np.flatnonzero(flags)
    np.bitwise_or.at(words, idx // 32, np.uint32(1) << (idx % 32).astype(np.uint32))
    gv.gvote_prune8(p, c, torch.from_numpy(words.view(np.int32)[None].copy()).cuda(), out, ws)
    assert gv.gvote_poll_status(ws) == 0 and int(out.kv_len[0, 0]) == idx.size
    for rows, first, last in ((K, (c.K, c.k_scale), (out.K, out.k_scale)), (V, (c.V, c.v_scale), (out.V, out.v_scale))):
        codes, scales = co.quantise(rows[0].double().numpy())
        got = read(c, *first, n)
        assert np.array_equal(got[0], codes, equal_nan=True) and np.array_equal(got[1], scales)
        want = co.quantise(co.values(codes, scales)[idx])
        got = read(out, *last, idx.size)
        assert np.array_equal(got[1], want[1]) and np.array_equal(got[0], want[0], equal_nan=True)
