"""The 8-bit cache, attention over it and the eviction by collected weight against their 64-bit oracle.

Codes, scales, lengths, masks and moved entries are compared exactly.  For the computed numbers, with products of stored
values exact in 32 bits or nearly so and sums in 32 bits, the bounds count the roundings:
  logits   each of the d_k products and additions is rounded once, chopped at worst (2^-23 relative to the sum of
           magnitudes): dl = d_k 2^-23 sum|q||k| / sqrt(d_k), plus 2^-22 |l| for the scaling
  weights  relative 2 dl + 2^-20: the logit's error in numerator and denominator, the exponential's few units, and
           2^-22 each for the sum and the log of the denominator
  out      half a step of bf16 (2^-8 |o|), then per term the weight's error, 2^-11 for its rounding to 16 bits before the
           product, and n 2^-24 for the sums in 32 bits, on sum w|v|
  lse      dl + 2^-20 + 2^-22 |lse|
  acc      weight error on the weights added, 2^-22 per term of the sum on the result"""
import math

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


def params(gv, hq, hkv, d, n_s=4):
    return gv.make_params(d_h=64, n_q_heads=hq, n_kv_heads=hkv, d_k=d, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=n_s, seed=0)


def cumulative(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def dev(x, dtype=None):
    t = torch.as_tensor(np.asarray(x))
    return (t if dtype is None else t.to(dtype)).cuda()


def bf16(rng, *shape, spread=0.0):
    x = rng.normal(size=shape)
    if spread:
        x = x * np.exp2(rng.uniform(-spread, spread, size=shape[:-1] + (1,)))
    return torch.from_numpy(x.astype(np.float32)).bfloat16()


def pack(gv, flags, cu):
    """Keep flags [hkv][total] -> mask words."""
    hkv, total = flags.shape
    m = np.zeros((hkv, gv.mask_row_words(total, len(cu) - 1)), dtype=np.uint32)
    for r in range(len(cu) - 1):
        off = gv.mask_word_offset(int(cu[r]), r)
        for h in range(hkv):
            n = np.flatnonzero(flags[h, cu[r]:cu[r + 1]])
            np.bitwise_or.at(m[h], off + n // 32, np.uint32(1) << (n % 32).astype(np.uint32))
    return dev(m.view(np.int32))


def strided(t, extra):
    """The same [heads, tokens, d] values as a window of a wider buffer, tokens outermost (head stride < token stride)."""
    H, T, d = t.shape
    buf = torch.zeros(T, H, d + extra, dtype=t.dtype, device=t.device)
    buf[:, :, :d] = t.transpose(0, 1)
    return buf[:, :, :d].transpose(0, 1)


def fill_cache(gv, p, lens, fill, rng, poison=True, spread=1.0):
    """A cache holding fill[r][h] random rows per head, and the oracle's (codes, scales) of them.  Rows behind the last
    hold the NaN code, scales behind the last block NaN."""
    cu = cumulative(lens)
    c = gv.alloc_cache8(p, cu)
    if poison:
        c.K.fill_(0x7f); c.V.fill_(0xff); c.k_scale.fill_(float("nan")); c.v_scale.fill_(float("nan"))
    held = {}
    for r in range(len(lens)):
        for h in range(p.n_kv_heads):
            n = fill[r][h]
            for w, (codes_t, scale_t) in enumerate(((c.K, c.k_scale), (c.V, c.v_scale))):
                x = bf16(rng, n, p.d_k, spread=spread).double().numpy()
                codes, scales = co.quantise(x)
                held[w, r, h] = codes, scales
                codes_t[h, cu[r]:cu[r] + n] = dev(codes, torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)
                b = gv.cache8_block_offset(int(cu[r]), r)
                scale_t[h, b:b + scales.size] = dev(scales, torch.float32)
    c.kv_len.copy_(dev(np.array(fill, dtype=np.int32).reshape(len(lens), p.n_kv_heads)))
    return c, held, cu


def read_cache(gv, c, w, r, h, n):
    codes, scale = (c.K, c.k_scale) if w == 0 else (c.V, c.v_scale)
    a = int(c.cu_seqlens[r])
    b = gv.cache8_block_offset(a, r)
    return (codes[h, a:a + n].view(torch.float8_e4m3fn).double().cpu().numpy(),
            scale[h, b:b + (n + 63) // 64].double().cpu().numpy())


def same(got, want):
    assert np.array_equal(got[0], want[0], equal_nan=True) and np.array_equal(got[1], want[1])


def workspace(gv, p, geom, total_q=0, max_q=0):
    """Behind the status word nothing of a workspace may matter: it holds NaNs there."""
    ws = gv.alloc_cache_workspace(p, *geom, total_q, max_q)
    ws[256:].fill_(0xff)
    return ws


# ----------------------------------------------------------------------------- store, prune
@gpu
@pytest.mark.parametrize("lens,hkv,d,density,strides", [
    ((1,), 1, 16, None, False), ((64,), 2, 64, 0.5, False), ((65, 0, 63, 128), 2, 80, 0.5, True),
    ((1000, 1, 333), 3, 128, 0.1, False), ((129, 700), 2, 256, 0.9, True), ((40000,), 1, 128, 0.3, False),
    ((300, 64), 2, 48, 0.0, False), ((9000, 2000), 1, 64, 0.002, False)])
@pytest.mark.parametrize("with_len", [False, True])
def test_store(gv, lens, hkv, d, density, strides, with_len):
    rng = np.random.default_rng(sum(lens) + d)
    p, cu, total = params(gv, hkv, hkv, d), cumulative(lens), sum(lens)
    K, V = bf16(rng, hkv, total, d, spread=6), bf16(rng, hkv, total, d, spread=6)
    Kd, Vd = (strided(t.cuda(), 8) if strides else t.cuda() for t in (K, V))
    flags = rng.random((hkv, total)) < density if density is not None else np.ones((hkv, total), dtype=bool)
    fill = [[int(rng.integers(0, n + 1)) if with_len else n for _ in range(hkv)] for n in lens]
    c = gv.alloc_cache8(p, cu)
    c.K.fill_(0x55); c.V.fill_(0x2a); c.k_scale.fill_(-1.0); c.v_scale.fill_(-2.0)
    if strides:                                                    # a destination with strides of its own, too
        c = gv.Cache8(strided(c.K, 16), strided(c.V, 16), c.k_scale, c.v_scale, c.cu_seqlens, c.kv_len, c.geom)
    acc, pos = rng.random((hkv, total)).astype(np.float32), rng.integers(0, 1 << 30, (hkv, total)).astype(np.int32)
    acc_out, pos_out = torch.full((hkv, total), -3.0).cuda(), torch.full((hkv, total), -4, dtype=torch.int32).cuda()
    ws = workspace(gv, p, c.geom)
    gv.gvote_store8(p, Kd, Vd, dev(cu), c.geom, c, ws, mask=None if density is None else pack(gv, flags, cu),
                    kv_len=dev(np.array(fill, dtype=np.int32).reshape(len(lens), hkv)) if with_len else None,
                    acc=dev(acc), acc_out=acc_out, token_pos=dev(pos), token_pos_out=pos_out)
    assert gv.gvote_poll_status(ws) == 0
    K64, V64 = K.double().numpy(), V.double().numpy()
    a, q = acc_out.cpu().numpy(), pos_out.cpu().numpy()
    for r, n in enumerate(lens):
        for h in range(hkv):
            idx = cu[r] + co.rows_of(flags[h, cu[r]:cu[r + 1]], fill[r][h])
            m = idx.size
            assert int(c.kv_len[r, h]) == m
            same(read_cache(gv, c, 0, r, h, m), co.quantise(K64[h, idx]))
            same(read_cache(gv, c, 1, r, h, m), co.quantise(V64[h, idx]))
            assert np.array_equal(a[h, cu[r]:cu[r] + m], acc[h, idx]) and np.array_equal(q[h, cu[r]:cu[r] + m], pos[h, idx])
            # behind the last row and the last block everything is as it was
            assert (c.K[h, cu[r] + m:cu[r + 1]] == 0x55).all() and (c.V[h, cu[r] + m:cu[r + 1]] == 0x2a).all()
            b0, b1 = (gv.cache8_block_offset(int(cu[i]), i) for i in (r, r + 1))
            if r + 1 < len(lens):
                assert (c.k_scale[h, b0 + (m + 63) // 64:b1] == -1).all()
            assert (a[h, cu[r] + m:cu[r + 1]] == -3).all() and (q[h, cu[r] + m:cu[r + 1]] == -4).all()


@gpu
def test_store_range_of_values_and_positions_of_a_first_store(gv):
    p = params(gv, 1, 1, 16)
    x = torch.zeros(1, 6 * 64, 16)
    x[0, 0:64] = 0.0
    x[0, 64:128, 0] = torch.tensor([2.0 ** -133, -(2.0 ** -127)] * 32)
    x[0, 128:192, 3] = 3.3895e38
    x[0, 130, 4] = -1.0
    x[0, 192, 0], x[0, 193, 1], x[0, 194, 2], x[0, 195, 3] = float("inf"), float("nan"), -float("inf"), 3.0
    x[0, 256:320] = torch.linspace(-448, 448, 1024).view(64, 16)
    x[0, 320:384] = -0.0
    K = x.bfloat16()
    c = gv.alloc_cache8(p, [0, 384])
    pos = torch.zeros(1, 384, dtype=torch.int32).cuda()
    ws = workspace(gv, p, c.geom)
    flags = np.ones((1, 384), dtype=bool)
    gv.gvote_store8(p, K.cuda(), K.cuda(), c.cu_seqlens, c.geom, c, ws, mask=pack(gv, flags, [0, 384]), token_pos_out=pos)
    same(read_cache(gv, c, 0, 0, 0, 384), co.quantise(K[0].double().numpy()))
    same(read_cache(gv, c, 1, 0, 0, 384), co.quantise(K[0].double().numpy()))
    assert np.array_equal(pos[0].cpu().numpy(), np.arange(384))


@gpu
@pytest.mark.parametrize("cap", [0, 1, 64, 100])
def test_store_drops_and_reports_rows_that_do_not_fit(gv, cap):
    rng = np.random.default_rng(cap)
    p = params(gv, 2, 2, 32)
    K, V = bf16(rng, 2, 200, 32), bf16(rng, 2, 200, 32)
    c = gv.alloc_cache8(p, [0, cap, cap + 130])
    cu = dev(cumulative((120, 80)))
    ws = workspace(gv, p, (2, max(200, cap + 130), max(130, cap)))
    gv.gvote_store8(p, K.cuda(), V.cuda(), cu, (2, 200, 120), c, ws)
    assert gv.gvote_poll_status(ws) == -3
    gv.gvote_clear_status(ws)
    assert gv.gvote_poll_status(ws) == 0
    for h in range(2):
        assert c.kv_len[:, h].tolist() == [min(cap, 120), 80]
        same(read_cache(gv, c, 0, 0, h, min(cap, 120)), co.quantise(K[h, :min(cap, 120)].double().numpy()))
        same(read_cache(gv, c, 1, 1, h, 80), co.quantise(V[h, 120:].double().numpy()))


@gpu
@pytest.mark.parametrize("lens,hkv,d,density", [((1,), 1, 16, 1.0), ((500, 64, 0, 1), 2, 128, 0.5), ((3000,), 3, 80, 0.2),
                                                ((200, 900), 2, 256, 0.9)])
def test_prune(gv, lens, hkv, d, density):
    rng = np.random.default_rng(sum(lens))
    p, total = params(gv, hkv, hkv, d), sum(lens)
    fill = [[int(rng.integers(n // 2, n + 1)) for _ in range(hkv)] for n in lens]
    src, held, cu = fill_cache(gv, p, lens, fill, rng, spread=8)
    flags = rng.random((hkv, total)) < density
    out_lens = [n + 7 for n in lens]                               # slabs of their own
    cu8 = cumulative(out_lens)
    out = gv.alloc_cache8(p, cu8)
    acc = rng.random((hkv, total)).astype(np.float32)
    acc_out = torch.zeros(hkv, int(cu8[-1])).cuda()
    ws = workspace(gv, p, out.geom)
    gv.gvote_prune8(p, src, pack(gv, flags, cu), out, ws, acc=dev(acc), acc_out=acc_out)
    assert gv.gvote_poll_status(ws) == 0
    for r in range(len(lens)):
        for h in range(hkv):
            idx = co.rows_of(flags[h, cu[r]:cu[r + 1]], fill[r][h])
            assert int(out.kv_len[r, h]) == idx.size
            for w in range(2):
                same(read_cache(gv, out, w, r, h, idx.size), co.quantise(co.values(*held[w, r, h])[idx]))
            assert np.array_equal(acc_out[h, cu8[r]:cu8[r] + idx.size].cpu().numpy(), acc[h, cu[r] + idx])


# ----------------------------------------------------------------------------- append
@gpu
@pytest.mark.parametrize("new,d,inplace", [((1, 1, 1, 1), 128, True), ((0, 3, 64, 65), 64, False), ((200, 0, 1, 700), 80, True),
                                           ((0, 0, 0, 0), 16, False), ((2, 130, 1, 1), 256, True)])
def test_append(gv, new, d, inplace):
    rng = np.random.default_rng(sum(new) + d)
    hkv, lens = 3, (1000, 300, 200, 1200)
    p = params(gv, hkv, hkv, d)
    fill = [[0, 64, 63], [1, 127, 128], [130, 65, 100], [500, 0, 448]]
    c, held, cu = fill_cache(gv, p, lens, fill, rng)
    total_new, cu_new = sum(new), cumulative(new)
    K, V = (bf16(rng, hkv, total_new, d, spread=4) for _ in range(2))      # some rows outgrow their block's scale
    acc, pos = torch.full((hkv, sum(lens)), 5.0).cuda(), torch.full((hkv, sum(lens)), -1, dtype=torch.int32).cuda()
    pos_new = dev(np.arange(total_new, dtype=np.int32) * 3 + 7)
    out = c.kv_len if inplace else torch.zeros_like(c.kv_len)
    ws = workspace(gv, p, c.geom)
    gv.gvote_append8(p, K.cuda(), V.cuda(), dev(cu_new), max(new), c, out, ws, acc=acc, token_pos=pos, pos_new=pos_new)
    assert gv.gvote_poll_status(ws) == 0
    for r in range(len(lens)):
        for h in range(hkv):
            n, m = fill[r][h], new[r]
            assert int(out[r, h]) == n + m and (inplace or int(c.kv_len[r, h]) == n)
            for w, X in enumerate((K, V)):
                want = co.append(*held[w, r, h], X[h, cu_new[r]:cu_new[r + 1]].double().numpy())
                same(read_cache(gv, c, w, r, h, n + m), want)
            a = acc[h, cu[r]:cu[r + 1]].cpu().numpy()
            assert (a[:n] == 5).all() and (a[n:n + m] == 0).all() and (a[n + m:] == 5).all()
            q = pos[h, cu[r]:cu[r + 1]].cpu().numpy()
            assert np.array_equal(q[n:n + m], np.arange(cu_new[r], cu_new[r + 1]) * 3 + 7) and (q[n + m:] == -1).all()
            assert (c.K[h, cu[r] + n + m:cu[r + 1]] == 0x7f).all()         # rows behind the last, as they were


@gpu
def test_append_one_by_one_and_a_full_slab(gv):
    rng = np.random.default_rng(3)
    p = params(gv, 2, 2, 64)
    c, held, cu = fill_cache(gv, p, (70, 10), [[0, 69], [10, 9]], rng)
    state = dict(held)
    ws = workspace(gv, p, c.geom)
    lens = {(r, h): [[0, 69], [10, 9]][r][h] for r in range(2) for h in range(2)}
    for step in range(3):
        K, V = (bf16(rng, 2, 2, 64, spread=5) for _ in range(2))
        gv.gvote_append8(p, K.cuda(), V.cuda(), dev(cumulative((1, 1))), 1, c, c.kv_len, ws)
        for (r, h), n in lens.items():
            if n < (70, 10)[r]:
                for w, X in enumerate((K, V)):
                    state[w, r, h] = co.append(*state[w, r, h], X[h, r:r + 1].double().numpy())
                lens[r, h] = n + 1
    assert gv.gvote_poll_status(ws) == -3                                   # three of the four heads ran full
    for (r, h), n in lens.items():
        assert int(c.kv_len[r, h]) == n
        for w in range(2):
            same(read_cache(gv, c, w, r, h, n), state[w, r, h])


# ----------------------------------------------------------------------------- attend
def check_attend(q, k, v, out, lse, acc_add=None, acc_in=None, acc_out=None):
    """One KV head of one request: q [n_q, g, d] float64, device results as float64 arrays."""
    n, d = k.shape
    o, l, w = co.attend(q, k, v)
    weights, _ = co.softmax_rows(q, k, q.shape[0])
    mag = np.einsum("igd,nd->ign", np.abs(q), np.abs(k)).max(initial=0.0) / math.sqrt(d)
    dl = d * 2.0 ** -23 * mag + 2.0 ** -22 * mag
    dw = 2 * dl + 2.0 ** -20
    a = np.einsum("ign,nd->igd", weights, np.abs(v))
    assert np.isfinite(out).all()
    assert (np.abs(out - o) <= 2.0 ** -8 * np.abs(o) + (dw + 2.0 ** -11 + n * 2.0 ** -24) * a).all()
    empty = np.isneginf(l)
    assert np.array_equal(np.isneginf(lse), empty) and (out[empty] == 0).all()
    assert (np.abs(lse[~empty] - l[~empty]) <= dl + 2.0 ** -20 + 2.0 ** -22 * np.abs(l[~empty])).all()
    if acc_out is not None:
        terms = q.shape[0] * q.shape[1] + 2
        assert (np.abs(acc_out - acc_in - w) <= dw * w + terms * 2.0 ** -22 * (w + np.abs(acc_in))).all()


def run_attend(gv, hq, hkv, d, lens, fill, n_q, seed=0, acc="separate", strides=False, q_scale=1.0, spread=1.0):
    rng = np.random.default_rng(seed)
    p, g = params(gv, hq, hkv, d), hq // hkv
    c, held, cu = fill_cache(gv, p, lens, fill, rng, spread=spread)
    if strides:
        c = gv.Cache8(strided(c.K, 16), strided(c.V, 16), c.k_scale, c.v_scale, c.cu_seqlens, c.kv_len, c.geom)
    tq, cq = sum(n_q), cumulative(n_q)
    Q = (bf16(rng, tq, hq, d).float() * q_scale).bfloat16()
    Qd, out = Q.cuda(), torch.full((tq, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    if strides:
        Qd, out = strided(Qd, 24), strided(out, 8)
    lse = torch.full((tq, hq), float("nan")).cuda()
    total = sum(lens)
    acc_in = (torch.from_numpy(rng.random((hkv, total)).astype(np.float32)) * 3).cuda()
    acc_out = {"separate": torch.full((hkv, total), -9.0).cuda(), "inplace": acc_in.clone(), None: None,
               "zero": torch.full((hkv, total), -9.0).cuda()}[acc]
    ws = workspace(gv, p, c.geom, tq, max(n_q))
    gv.gvote_attend8(p, Qd, dev(cq), max(n_q), c, out, ws, lse=lse,
                     acc={"separate": acc_in, "inplace": acc_out, None: None, "zero": None}[acc], acc_out=acc_out)
    assert gv.gvote_poll_status(ws) == 0
    base = np.zeros((hkv, total)) if acc == "zero" else acc_in.double().cpu().numpy()
    Q64, o64, l64 = Q.double().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    got = None if acc is None else acc_out.double().cpu().numpy()
    for r in range(len(lens)):
        t = slice(cq[r], cq[r + 1])
        for h in range(hkv):
            hs, n = slice(h * g, (h + 1) * g), fill[r][h]
            k, v = co.values(*held[0, r, h]), co.values(*held[1, r, h])
            s = slice(cu[r], cu[r] + n)
            check_attend(Q64[t, hs], k, v, o64[t, hs], l64[t, hs], None, base[h, s], None if got is None else got[h, s])
            if got is not None:                                    # slots without a row, as they were
                rest = got[h, cu[r] + n:cu[r + 1]]
                assert np.array_equal(rest, base[h, cu[r] + n:cu[r + 1]] if acc == "inplace" else np.full(rest.shape, -9.0))
    return c, Qd, out, lse


@gpu
@pytest.mark.parametrize("hq,hkv,d,lens,fill,n_q", [
    (1, 1, 16, (1,), [[1]], (1,)),
    (8, 2, 64, (512,), [[512, 300]], (1,)),
    (4, 1, 128, (64, 65, 63, 1), [[64], [65], [63], [0]], (1, 1, 1, 1)),
    (28, 4, 128, (1500, 700), [[1500, 0, 1, 999], [700, 640, 64, 333]], (1, 1)),
    (6, 3, 80, (300, 0, 40), [[300, 5, 64], [0, 0, 0], [40, 39, 2]], (2, 3, 5)),
    (5, 5, 256, (260, 129), [[260, 100, 3, 255, 257], [129, 128, 127, 0, 1]], (1, 4)),
    (32, 8, 128, (4096,), [[4096, 100, 2000, 0, 64, 65, 1, 3333]], (5,)),
    (16, 1, 96, (900,), [[900]], (9,)),
    (24, 2, 64, (333,), [[320, 31]], (32,)),
    (8, 8, 128, (5000, 3), [[5000, 1, 2, 3, 4, 5, 6, 7], [3, 3, 2, 2, 1, 1, 0, 0]], (1, 0)),
])
def test_attend(gv, hq, hkv, d, lens, fill, n_q):
    run_attend(gv, hq, hkv, d, lens, fill, n_q, seed=sum(lens) + d)


@gpu
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("hq,hkv,n_q", [(3, 1, 1), (5, 1, 1), (9, 1, 1), (16, 1, 1), (5, 1, 4), (8, 1, 3), (7, 1, 4), (11, 1, 3), (128, 1, 2)])
def test_attend_row_counts(gv, hq, hkv, n_q, d):
    """Every way the query rows are dealt to the softmax groups: 1 to 4, 8, 12, 16, 20, 24, 32 rows, and more than one
    group of 32, over several requests of very different length."""
    run_attend(gv, hq, hkv, d, (700, 1, 130, 4000, 260), [[700], [1], [129], [3333], [256]], (n_q, 1, n_q, n_q, 0), seed=hq + n_q)


@gpu
@pytest.mark.parametrize("n_q", [1, 2, 5])
def test_attend_fewer_tiles_than_ctas(gv, n_q):
    """Long slabs that hold a few rows: the grid is sized for the slabs, most of its CTAs have nothing."""
    for rows in ((200, 129, 130), (1, 0, 300), (128, 257, 5), (0, 0, 1), (900, 385, 1)):
        run_attend(gv, 4, 2, 64, (2000, 2000, 1500), [[n, max(n - n_q, 0)] for n in rows], (n_q, 1, n_q), seed=27)


@gpu
def test_attend_many_short_requests(gv):
    """More entries than one launch takes (1024), most of them of a single tile or empty, so that a CTA's tiles change
    their head at every step."""
    rng = np.random.default_rng(20)
    lens = tuple(int(x) for x in rng.integers(1, 200, size=150))
    fill = [[int(rng.integers(0, n + 1)) for _ in range(8)] for n in lens]
    run_attend(gv, 16, 8, 64, lens, fill, tuple(int(x) for x in rng.integers(0, 4, size=150)), seed=21)


@gpu
@pytest.mark.parametrize("hq,d,n_q", [(4, 64, 1), (3, 256, 2)])
def test_attend_one_long_request_among_many_short_ones(gv, hq, d, n_q):
    """Most rows are merged from a few parts, the long request's from more than a hundred."""
    lens = (20, 3) * 40 + (30000,) + (1, 20, 0) * 30
    run_attend(gv, hq, 1, d, lens, [[n] for n in lens], tuple(min(n_q, n) for n in lens), seed=28)


@gpu
def test_a_workspace_serves_every_smaller_call(gv):
    p = params(gv, 7, 1, 64)
    rng = np.random.default_rng(22)
    c, held, cu = fill_cache(gv, p, (500, 300), [[500], [300]], rng)
    ws = workspace(gv, p, c.geom, 64, 32)
    K = bf16(rng, 1, 800, 64).cuda()
    for n_q in (1, 2, 3, 4, 5, 9, 32):
        for m in (n_q, 0):
            Q = bf16(rng, n_q + m, 7, 64).cuda()
            cq = dev(cumulative((n_q, m)))
            gv.gvote_attend8(p, Q, cq, n_q, c, torch.empty_like(Q), ws, acc_out=torch.zeros(1, 800).cuda())
            gv.gvote_accumulate(p, Q, cq, n_q, K, c.cu_seqlens, c.geom, torch.zeros(1, 800).cuda(), ws)
    assert gv.gvote_poll_status(ws) == 0


@gpu
@pytest.mark.parametrize("acc", ["inplace", "zero", None])
def test_attend_weights_in_place_from_zero_and_not_at_all(gv, acc):
    run_attend(gv, 8, 2, 128, (700, 70), [[700, 321], [70, 0]], (2, 1), seed=5, acc=acc)


@gpu
def test_attend_strided_tensors(gv):
    run_attend(gv, 12, 4, 64, (400, 130), [[400, 64, 200, 7], [130, 129, 0, 64]], (3, 1), seed=6, strides=True)


@gpu
@pytest.mark.parametrize("q_scale,spread", [(30.0, 1.0), (1e-3, 6.0), (4.0, 12.0)])
def test_attend_sharp_and_flat_rows_and_blocks_of_very_different_scale(gv, q_scale, spread):
    run_attend(gv, 8, 2, 128, (1000,), [[1000, 777]], (2,), seed=8, q_scale=q_scale, spread=spread)


@gpu
def test_attend_one_row_holds_all_weight_and_its_value_is_small(gv):
    """A block of large values with next to no weight beside a block of tiny values with all of it."""
    p = params(gv, 2, 1, 64)
    K, V = torch.zeros(1, 256, 64), torch.zeros(1, 256, 64)
    K[0, :, 0] = -100.0
    K[0, 200, 0] = 100.0
    V[0, :128] = 1e30
    V[0, 128:] = 1e-20
    c = gv.alloc_cache8(p, [0, 256])
    ws = workspace(gv, p, c.geom, 1, 1)
    gv.gvote_store8(p, K.bfloat16().cuda(), V.bfloat16().cuda(), c.cu_seqlens, c.geom, c, ws)
    Q = torch.zeros(1, 2, 64)
    Q[0, 0, 0], Q[0, 1, 0] = 8.0, 0.25
    out, lse = torch.zeros(1, 2, 64, dtype=torch.bfloat16).cuda(), torch.zeros(1, 2).cuda()
    gv.gvote_attend8(p, Q.bfloat16().cuda(), dev(cumulative((1,))), 1, c, out, ws, lse=lse)
    k, v = (co.values(*read_cache(gv, c, w, 0, 0, 256)) for w in range(2))
    check_attend(Q.bfloat16().double().numpy(), k, v, out.double().cpu().numpy(), lse.double().cpu().numpy())


@gpu
def test_attend_shows_a_nan_that_a_seen_row_holds(gv):
    rng = np.random.default_rng(9)
    p = params(gv, 2, 2, 64)
    c, _, cu = fill_cache(gv, p, (200,), [[200, 150]], rng)
    c.V[0, 100, 5] = 0x7f
    c.K[1, 149, 3] = 0xff
    Q = bf16(rng, 2, 2, 64).cuda()
    out = torch.zeros(2, 2, 64, dtype=torch.bfloat16).cuda()
    ws = workspace(gv, p, c.geom, 2, 2)
    gv.gvote_attend8(p, Q, dev(cumulative((2,))), 2, c, out, ws)
    nan = out.isnan().cpu()
    assert nan[:, 0, 5].all() and nan[:, 0].sum() == 2             # one channel of the value, for both tokens
    assert nan[1, 1].all() and not nan[0, 1].any()                 # the key's row is hidden from the first token


@gpu
def test_attend_hides_a_nan_from_the_tokens_that_do_not_see_its_row(gv):
    """The last token's own value is NaN in one channel: it must show in the last token's output and in no other."""
    rng = np.random.default_rng(14)
    p = params(gv, 4, 2, 80)
    c, held, cu = fill_cache(gv, p, (300, 129), [[300, 200], [129, 5]], rng)
    c.V[0, 299, 7] = 0xff                                              # request 0, head 0, last row
    c.V[1, cu[1] + 3, 79] = 0x7f                                       # request 1, head 1, the last row but one
    Q = bf16(rng, 6, 4, 80)
    out, acc = torch.zeros(6, 4, 80, dtype=torch.bfloat16).cuda(), torch.zeros(2, 429).cuda()
    ws = workspace(gv, p, c.geom, 6, 3)
    for _ in range(2):                                                 # (the second call finds no mark of the first)
        gv.gvote_attend8(p, Q.cuda(), dev(cumulative((3, 3))), 3, c, out, ws, acc_out=acc)
        nan = out.isnan().cpu()
        assert nan[2, 0:2, 7].all() and nan[4:6, 2:4, 79].all() and nan.sum() == 2 + 4
        assert torch.isfinite(acc).all()
    o, _, _ = co.attend(Q[0:3, 0:2].double().numpy(), co.values(*held[0, 0, 0]), co.values(*held[1, 0, 0]))
    assert np.allclose(out[:2, 0:2].double().cpu().numpy(), o[:2], rtol=2.0 ** -7, atol=2.0 ** -7)


@gpu
def test_attend_is_deterministic_and_works_on_another_stream_and_in_a_graph(gv):
    rng = np.random.default_rng(10)
    p = params(gv, 8, 2, 128)
    c, _, cu = fill_cache(gv, p, (3000, 500), [[3000, 1111], [500, 64]], rng)
    Q = bf16(rng, 3, 8, 128).cuda()
    cq = dev(cumulative((2, 1)))
    ws = workspace(gv, p, c.geom, 3, 2)
    first = None
    for _ in range(3):
        out, acc = torch.zeros(3, 8, 128, dtype=torch.bfloat16).cuda(), torch.zeros(2, 3500).cuda()
        gv.gvote_attend8(p, Q, cq, 2, c, out, ws, acc_out=acc)
        first = first or (out.clone(), acc.clone())
        assert torch.equal(out, first[0]) and torch.equal(acc, first[1])
    s = torch.cuda.Stream()
    out, acc = torch.zeros_like(first[0]), torch.zeros_like(first[1])
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        gv.gvote_attend8(p, Q, cq, 2, c, out, ws, acc_out=acc)
    s.synchronize()
    assert torch.equal(out, first[0]) and torch.equal(acc, first[1])
    graphs = []                                                    # two graphs share the workspace, replayed in turn
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        o2, a2 = torch.zeros_like(first[0]), torch.zeros_like(first[1])
        with torch.cuda.graph(g):
            gv.gvote_attend8(p, Q, cq, 2, c, o2, ws, acc_out=a2)
        graphs.append((g, o2, a2))
    for _ in range(2):
        for g, o2, a2 in graphs:
            o2.zero_(); a2.zero_()
            g.replay()
    torch.cuda.synchronize()
    for _, o2, a2 in graphs:
        assert torch.equal(o2, first[0]) and torch.equal(a2, first[1])


@gpu
def test_rows_beyond_four_gigabytes_of_codes(gv):
    """A slab that starts past 2^32 bytes of the code arrays, and one head stride past it."""
    big = (1 << 25) + 77
    rng = np.random.default_rng(11)
    p = params(gv, 2, 2, 128)
    lens, fill = (big, 130), [[3, 0], [130, 67]]
    c, held, cu = fill_cache(gv, p, lens, fill, rng, poison=False)
    Q = bf16(rng, 2, 2, 128)
    out, lse = torch.zeros(2, 2, 128, dtype=torch.bfloat16).cuda(), torch.zeros(2, 2).cuda()
    ws = workspace(gv, p, c.geom, 2, 1)
    new = [bf16(rng, 2, 2, 128) for _ in range(2)]
    gv.gvote_append8(p, new[0].cuda(), new[1].cuda(), dev(cumulative((1, 0))), 1, c, c.kv_len, ws)
    gv.gvote_attend8(p, Q.cuda(), dev(cumulative((1, 1))), 1, c, out, ws, lse=lse)
    for r in range(2):
        for h in range(2):
            kv = [co.append(*held[w, r, h], new[w][h, :1 - r].double().numpy()) for w in range(2)]
            check_attend(Q[r:r + 1, h:h + 1].double().numpy(), co.values(*kv[0]), co.values(*kv[1]),
                         out[r:r + 1, h:h + 1].double().cpu().numpy(), lse[r:r + 1, h:h + 1].double().cpu().numpy())


# ----------------------------------------------------------------------------- accumulate
def run_accumulate(gv, hq, hkv, d, lens, n_q, fill=None, given_lse=False, acc="separate", strides=False, seed=0, q_scale=1.5):
    rng = np.random.default_rng(seed)
    p, g, total = params(gv, hq, hkv, d), hq // hkv, sum(lens)
    cu, cq, tq = cumulative(lens), cumulative(n_q), sum(n_q)
    K = bf16(rng, hkv, total, d)
    Q = (bf16(rng, tq, hq, d).float() * q_scale).bfloat16()
    fill = fill or [[n] * hkv for n in lens]
    kv = dev(np.array(fill, dtype=np.int32).reshape(len(lens), hkv))
    K_dirty = K.clone()
    for r, n in enumerate(lens):
        for h in range(hkv):
            K_dirty[h, cu[r] + fill[r][h]:cu[r + 1]] = float("nan")          # behind the rows that count
    Kd, Qd = K_dirty.cuda(), Q.cuda()
    if strides:
        Kd, Qd = strided(Kd, 8), strided(Qd, 16)
    want, lse = np.zeros((hkv, total)), np.full((tq, hq), -np.inf)
    tol = np.zeros((hkv, total))
    acc_in = rng.random((hkv, total)).astype(np.float32)
    base = np.zeros((hkv, total)) if acc == "zero" else acc_in.astype(np.float64)
    for r in range(len(lens)):
        for h in range(hkv):
            n = fill[r][h]
            q, k = Q[cq[r]:cq[r + 1], h * g:(h + 1) * g].double().numpy(), K[h, cu[r]:cu[r] + n].double().numpy()
            w, l = co.softmax_rows(q, k, n_q[r])
            lse[cq[r]:cq[r + 1], h * g:(h + 1) * g] = l
            s = slice(cu[r], cu[r] + n)
            want[h, s] = w.sum(axis=(0, 1))
            mag = (np.abs(q).reshape(-1, d) @ np.abs(k).T).max(initial=0.0) / math.sqrt(d)
            dl = d * 2.0 ** -23 * mag + 2.0 ** -22 * mag
            # the log-sum-exp enters the exponent in 32 bits: 2^-23 |lse|
            lmax = np.abs(l[np.isfinite(l)]).max(initial=0.0)
            tol[h, s] = (2 * dl + 2.0 ** -20 + 2.0 ** -21 * lmax + (n_q[r] * g + 2) * 2.0 ** -24) * want[h, s] + 2.0 ** -22 * np.abs(base[h, s])
    acc_t = dev(acc_in)
    out = acc_t if acc == "inplace" else torch.full((hkv, total), -9.0).cuda()
    ws = workspace(gv, p, (len(lens), total, max(lens)), tq, max(n_q))
    gv.gvote_accumulate(p, Qd, dev(cq), max(n_q), Kd, dev(cu), (len(lens), total, max(lens)), out, ws,
                        acc=None if acc == "zero" else acc_t, lse=dev(lse, torch.float32) if given_lse else None, kv_len=kv)
    assert gv.gvote_poll_status(ws) == 0
    got = out.double().cpu().numpy()
    for r in range(len(lens)):
        for h in range(hkv):
            s = slice(cu[r], cu[r] + fill[r][h])
            assert (np.abs(got[h, s] - base[h, s] - want[h, s]) <= tol[h, s]).all()
            rest = slice(cu[r] + fill[r][h], cu[r + 1])
            assert np.array_equal(got[h, rest], base[h, rest] if acc == "inplace" else np.full(got[h, rest].shape, -9.0))


@gpu
@pytest.mark.parametrize("hq,hkv,d,lens,n_q", [
    (1, 1, 16, (1,), (1,)), (8, 2, 64, (512,), (512,)), (8, 2, 64, (512, 100), (1, 0)), (4, 1, 128, (129, 127), (129, 64)),
    (28, 4, 128, (700,), (32,)), (14, 2, 128, (300,), (300,)), (6, 3, 80, (257, 0, 33), (257, 0, 20)),
    (5, 5, 256, (400,), (130,)), (16, 1, 96, (1000,), (1000,)), (32, 8, 128, (1200,), (40,)), (2, 2, 48, (60, 5), (64, 9)),
    (128, 1, 64, (90,), (70,)), (4, 2, 128, (2500,), (2500,)), (4, 2, 192, (3000,), (5,)),
])
def test_accumulate(gv, hq, hkv, d, lens, n_q):
    run_accumulate(gv, hq, hkv, d, lens, n_q, seed=sum(lens) + d)


@gpu
@pytest.mark.parametrize("kw", [dict(given_lse=True), dict(acc="inplace"), dict(acc="zero"), dict(strides=True),
                                dict(fill=[[300, 1], [0, 129]]), dict(fill=[[31, 300], [200, 7]], given_lse=True), dict(q_scale=12.0)])
def test_accumulate_variants(gv, kw):
    run_accumulate(gv, 8, 2, 128, (300, 200), (40, 200), seed=4, **kw)


# ----------------------------------------------------------------------------- evict
@gpu
@pytest.mark.parametrize("lens,hkv,n_recent,n_s,kind", [
    ((1,), 1, 0, 0, "random"), ((64, 65, 0, 1), 2, 3, 4, "random"), ((1000, 33), 3, 32, 4, "ties"), ((5000,), 2, 0, 0, "equal"),
    ((40000, 20), 2, 500, 4, "random"), ((3000,), 2, 10000, 4, "random"), ((3000, 700), 2, 0, 4, "signs"), ((2000,), 3, 5, 4, "nan"),
    ((131072,), 1, 64, 4, "ties"), ((200000,), 1, 64, 4, "random"), ((70000, 6000, 33000), 2, 64, 4, "random")])
def test_evict(gv, lens, hkv, n_recent, n_s, kind):
    rng = np.random.default_rng(sum(lens))
    p, cu, total = params(gv, hkv, hkv, 16, n_s=n_s), cumulative(lens), sum(lens)
    acc = np.exp(rng.normal(size=(hkv, total)) * 3).astype(np.float32)
    if kind == "ties":
        acc = rng.integers(0, 5, (hkv, total)).astype(np.float32)
    if kind == "equal":
        acc[:] = 0.25
    if kind == "signs":
        acc = rng.choice(np.array([0.0, -0.0, 1e-45, -1e-45, np.inf, -np.inf, 1.0], dtype=np.float32), (hkv, total))
    if kind == "nan":
        acc[rng.random((hkv, total)) < 0.5] = np.nan
    for share, with_len in ((0.0, False), (0.3, False), (0.7, True), (1.0, True), (1.5, False)):
        fill = [[int(rng.integers(0, n + 1)) if with_len else n for _ in range(hkv)] for n in lens]
        keep = np.array([[int(n * share) - (h == 1) for h in range(hkv)] for n in lens], dtype=np.int32).reshape(len(lens), hkv)
        mask = torch.full((hkv, gv.mask_row_words(total, len(lens))), -1, dtype=torch.int32).cuda()
        budget = torch.full((len(lens), hkv), -1, dtype=torch.int32).cuda()
        geom = (len(lens), total, max(lens))
        gv.gvote_evict(p, dev(acc), dev(cu), geom, dev(keep), n_recent, mask, budget, workspace(gv, p, geom),
                       kv_len=dev(np.array(fill, dtype=np.int32).reshape(len(lens), hkv)) if with_len else None)
        m, b = mask.cpu().numpy(), budget.cpu().numpy()
        for r, n in enumerate(lens):
            for h in range(hkv):
                want = np.zeros((n + 31) // 32 * 32, dtype=bool)
                want[:fill[r][h]] = co.evict(acc[h, cu[r]:cu[r] + fill[r][h]], int(keep[r, h]), n_recent, n_s)
                got = gv.unpack_mask(m[h], gv.mask_word_offset(int(cu[r]), r), want.size)
                assert np.array_equal(got, want), (share, r, h)              # padding bits are zero, too
                assert b[r, h] == want.sum()


@gpu
def test_evict_rows_that_outgrow_shared_memory(gv):
    """400000 rows: eight shares of 50000, more than a CTA stages."""
    rng = np.random.default_rng(23)
    p, n = params(gv, 2, 2, 16), 400000
    geom = (1, n, n)
    for acc, keep in ((np.exp(rng.normal(size=(2, n)) * 3), [123457, 399990]), (rng.integers(0, 3, (2, n)), [200001, 17])):
        acc = acc.astype(np.float32)
        mask = torch.full((2, gv.mask_row_words(n, 1)), -1, dtype=torch.int32).cuda()
        budget = torch.zeros(1, 2, dtype=torch.int32).cuda()
        gv.gvote_evict(p, dev(acc), dev(cumulative((n,))), geom, dev(np.array([keep], dtype=np.int32)), 8, mask, budget,
                       workspace(gv, p, geom))
        m = mask.cpu().numpy()
        for h in range(2):
            assert np.array_equal(gv.unpack_mask(m[h], 0, n), co.evict(acc[h], keep[h], 8, 4))
            assert budget[0, h] == keep[h]


# ----------------------------------------------------------------------------- together
def whole_flow(gv, p, t):
    """A prompt's weights, eviction, store, two tokens, eviction and prune: every entry point once, into t's buffers."""
    gv.gvote_accumulate(p, t.Q, t.cu_q, 300, t.K, t.cu, t.geom, t.acc, t.ws)
    gv.gvote_evict(p, t.acc, t.cu, t.geom, t.keep, 8, t.mask, t.budget, t.ws)
    gv.gvote_store8(p, t.K, t.V, t.cu, t.geom, t.c, t.ws, mask=t.mask, acc=t.acc, acc_out=t.acc8, token_pos_out=t.pos8)
    gv.gvote_append8(p, t.kn, t.vn, t.cu_new, 2, t.c, t.c.kv_len, t.ws, acc=t.acc8, token_pos=t.pos8, pos_new=t.pos_new)
    gv.gvote_attend8(p, t.qn, t.cu_new, 2, t.c, t.out, t.ws, acc=t.acc8, acc_out=t.acc8)
    gv.gvote_evict(p, t.acc8, t.c.cu_seqlens, t.c.geom, t.keep2, 4, t.mask8, t.budget, t.ws, kv_len=t.c.kv_len)
    gv.gvote_prune8(p, t.c, t.mask8, t.c2, t.ws, acc=t.acc8, acc_out=t.acc2, token_pos=t.pos8, token_pos_out=t.pos2)
    return [x.clone() for x in (t.acc, t.mask, t.out, t.acc2, t.pos2, t.c2.kv_len, t.c2.K, t.c2.V, t.c2.k_scale, t.c2.v_scale)]


def flow_tensors(gv, p, hq, hkv, d):
    from types import SimpleNamespace
    rng = np.random.default_rng(24)
    lens, caps = (1000, 41, 300), (600, 50, 220)
    cu, cu8 = cumulative(lens), cumulative(caps)
    t = SimpleNamespace(geom=(3, 1341, 1000), cu=dev(cu), cu_q=dev(cumulative((300, 41, 300))), cu_new=dev(cumulative((1, 2, 0))))
    t.K, t.V, t.Q = bf16(rng, hkv, 1341, d).cuda(), bf16(rng, hkv, 1341, d).cuda(), bf16(rng, 641, hq, d).cuda()
    t.kn, t.vn, t.qn = bf16(rng, hkv, 3, d).cuda(), bf16(rng, hkv, 3, d).cuda(), bf16(rng, 3, hq, d).cuda()
    t.keep = dev(np.tile(np.array([[500], [40], [100]], dtype=np.int32), (1, hkv)))
    t.keep2 = dev(np.tile(np.array([[77], [30], [100]], dtype=np.int32), (1, hkv)))
    t.pos_new = dev(np.array([1000, 41, 42], dtype=np.int32))
    t.c, t.c2 = gv.alloc_cache8(p, cu8), gv.alloc_cache8(p, cu8)
    t.acc, t.acc8, t.acc2 = (torch.zeros(hkv, n).cuda() for n in (1341, 870, 870))
    t.pos8, t.pos2 = (torch.zeros(hkv, 870, dtype=torch.int32).cuda() for _ in range(2))
    t.mask, t.mask8 = (torch.zeros(hkv, gv.mask_row_words(n, 3), dtype=torch.int32).cuda() for n in (1341, 870))
    t.budget = torch.zeros(3, hkv, dtype=torch.int32).cuda()
    t.out = torch.zeros(3, hq, d, dtype=torch.bfloat16).cuda()
    t.ws = workspace(gv, p, t.geom, 641, 300)
    return t


@gpu
def test_the_whole_flow_on_another_stream_and_in_a_graph(gv):
    """The same bits eagerly, on a side stream, and from a captured graph that is replayed; two calls at once with a
    workspace each."""
    p = params(gv, 6, 2, 64)
    t = flow_tensors(gv, p, 6, 2, 64)
    want = whole_flow(gv, p, t)
    others = [flow_tensors(gv, p, 6, 2, 64) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in others]
    torch.cuda.synchronize()
    for u, s in zip(others, streams):
        with torch.cuda.stream(s):
            for _ in range(3):
                got = whole_flow(gv, p, u)
            u.got = got
    torch.cuda.synchronize()
    for u in others:
        assert all(torch.equal(a, b) for a, b in zip(u.got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = whole_flow(gv, p, t)
    for _ in range(2):
        for x in (t.acc, t.acc8, t.acc2, t.out, t.c2.K, t.c2.V):
            x.zero_()
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(captured, want))
    assert all(gv.gvote_poll_status(u.ws) == 0 for u in (t, *others))


@gpu
def test_slabs_that_do_not_start_at_slot_zero(gv):
    """The later requests of a batch by a view of its boundaries: their results, and nothing written before them."""
    rng = np.random.default_rng(25)
    p, lens = params(gv, 4, 2, 64), (777, 500, 130)
    cu, total = cumulative(lens), 1407
    K, V, Q = bf16(rng, 2, total, 64).cuda(), bf16(rng, 2, total, 64).cuda(), bf16(rng, total, 4, 64).cuda()
    full, part = dev(cu), dev(cu[1:])
    flags = rng.random((2, total)) < 0.4
    for n_q in (lens, (777, 3, 130)):                                # (the first request's tokens: not looked at)
        cq = cumulative(n_q)
        geoms = ((3, total, 777), (2, total, 500))
        acc = [torch.full((2, total), -1.0).cuda() for _ in range(2)]
        ws = workspace(gv, p, geoms[0], int(cq[-1]), 777)
        for a, cu_d, cq_d, geom in zip(acc, (full, part), (dev(cq), dev(cq[1:])), geoms):
            gv.gvote_accumulate(p, Q[:cq[-1]], cq_d, 777, K, cu_d, geom, a, ws)
        assert (acc[1][:, :777] == -1).all() and (acc[0] >= 0).all()
        assert torch.allclose(acc[0][:, 777:], acc[1][:, 777:], rtol=1e-5, atol=0)
    acc1 = torch.full((2, total), -1.0).cuda()                       # one request, behind others
    gv.gvote_accumulate(p, Q, dev(cu[2:]), 130, K, dev(cu[2:]), (1, total, 130), acc1, ws)
    gv.gvote_accumulate(p, Q, full, 777, K, full, (3, total, 777), acc[0], ws)
    assert (acc1[:, :1277] == -1).all() and torch.allclose(acc[0][:, 1277:], acc1[:, 1277:], rtol=1e-5, atol=0)
    for masked in (False, True):
        caches = [gv.alloc_cache8(p, cu), gv.alloc_cache8(p, cu)]
        b = gv.Cache8(*(getattr(caches[1], n) for n in ("K", "V")), *(torch.zeros(2, gv.cache8_row_blocks(total, 2)).cuda() for _ in range(2)),
                      part, torch.zeros(2, 2, dtype=torch.int32).cuda(), (2, total, 500))
        caches[1] = b
        for c, cu_h, cu_d, geom in zip(caches, (cu, cu[1:]), (full, part), ((3, total, 777), (2, total, 500))):
            gv.gvote_store8(p, K, V, cu_d, geom, c, ws, mask=pack(gv, flags, cu_h) if masked else None)
        assert (b.K[:, :777] == 0).all() and torch.equal(b.K[:, 777:], caches[0].K[:, 777:])
        assert torch.equal(b.V[:, 777:], caches[0].V[:, 777:]) and torch.equal(b.kv_len, caches[0].kv_len[1:])
        outs = []
        for c, cq in zip(caches, (cumulative((1, 1, 1)), np.array([1, 2, 3], dtype=np.int32))):
            out, a = torch.zeros(3, 4, 64, dtype=torch.bfloat16).cuda(), torch.zeros(2, total).cuda()
            gv.gvote_attend8(p, Q[:3], dev(cq), 1, c, out, ws, acc_out=a)
            outs.append((out, a))
        assert torch.allclose(outs[0][0][1:].float(), outs[1][0][1:].float(), rtol=2.0 ** -6, atol=2.0 ** -8)
        assert (outs[1][0][0] == 0).all() and (outs[1][1][:, :777] == 0).all()
        assert torch.allclose(outs[0][1][:, 777:], outs[1][1][:, 777:], rtol=1e-4, atol=1e-9)
    assert gv.gvote_poll_status(ws) == 0


@gpu
def test_attend_reports_a_request_of_more_tokens_than_announced(gv):
    rng = np.random.default_rng(26)
    p = params(gv, 4, 2, 64)
    c, _, _ = fill_cache(gv, p, (300, 200), [[300, 300], [200, 200]], rng)
    ws = workspace(gv, p, c.geom, 6, 2)
    Q = bf16(rng, 6, 4, 64).cuda()
    out = torch.zeros_like(Q)
    gv.gvote_attend8(p, Q, dev(cumulative((2, 4))), 2, c, out, ws, acc_out=torch.zeros(2, 500).cuda())
    assert gv.gvote_poll_status(ws) == -1
    assert (out[4:] == 0).all()                                      # the excess is left alone


@gpu
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (14, 2, 128)])
def test_prompt_then_tokens_then_eviction(gv, hq, hkv, d):
    """As an engine uses them: weights of the prompt's last tokens, eviction, the rows into the 8-bit cache, tokens
    appended and attended to with the weights kept up, the full cache pruned again, and on."""
    rng = np.random.default_rng(12)
    lens, g = (300, 41), hq // hkv
    p, cu, batch = params(gv, hq, hkv, d), cumulative((300, 41)), 2
    total = int(cu[-1])
    K, V = (bf16(rng, hkv, total, d) for _ in range(2))
    window = (24, 24)
    Qw = bf16(rng, 48, hq, d)
    geom = (batch, total, max(lens))
    cu_d = dev(cu)
    ws = workspace(gv, p, geom, 48, 24)
    acc0 = torch.zeros(hkv, total).cuda()
    gv.gvote_accumulate(p, Qw.cuda(), dev(cumulative(window)), 24, K.cuda(), cu_d, geom, acc0, ws)
    keep = dev(np.array([[100, 60], [41, 20]], dtype=np.int32))
    mask = torch.zeros(hkv, gv.mask_row_words(total, batch), dtype=torch.int32).cuda()
    budget = torch.zeros(batch, hkv, dtype=torch.int32).cuda()
    gv.gvote_evict(p, acc0, cu_d, geom, keep, 8, mask, budget, ws)
    cu8 = cumulative((110, 48))
    c = gv.alloc_cache8(p, cu8)
    acc = torch.zeros(hkv, 158).cuda()
    pos = torch.zeros(hkv, 158, dtype=torch.int32).cuda()
    ws8 = workspace(gv, p, geom, 2, 1)
    gv.gvote_store8(p, K.cuda(), V.cuda(), cu_d, geom, c, ws8, mask=mask, acc=acc0, acc_out=acc, token_pos_out=pos)
    # the oracle alongside: the device's own weights decide what stays (they agree to rounding, selection is exact on them)
    a0 = acc0.cpu().numpy()
    codes, weights, where = {}, {}, {}
    for r in range(batch):
        for h in range(hkv):
            q = Qw[24 * r:24 * r + 24, h * g:(h + 1) * g].double().numpy()
            want = co.collected(q, K[h, cu[r]:cu[r + 1]].double().numpy())
            assert np.allclose(a0[h, cu[r]:cu[r + 1]], want, rtol=1e-4, atol=0)
            idx = np.flatnonzero(co.evict(a0[h, cu[r]:cu[r + 1]], int(keep[r, h]), 8, 4))
            assert np.array_equal(pos[h, cu8[r]:cu8[r] + idx.size].cpu().numpy(), idx)
            for w, X in enumerate((K, V)):
                codes[w, r, h] = co.quantise(X[h, cu[r] + idx].double().numpy())
            weights[r, h], where[r, h] = a0[h, cu[r] + idx].astype(np.float64), idx
    for step in range(14):
        k_new, v_new = (bf16(rng, hkv, batch, d, spread=2) for _ in range(2))
        q_new = bf16(rng, batch, hq, d)
        one = dev(cumulative((1, 1)))
        if step == 7:                                              # request 1 runs full: evict in both, prune
            n_now = c.kv_len.cpu().numpy()
            keep2 = dev(np.minimum(n_now, [[50], [30]]).astype(np.int32))
            mask8 = torch.zeros(hkv, gv.mask_row_words(158, batch), dtype=torch.int32).cuda()
            gv.gvote_evict(p, acc, c.cu_seqlens, c.geom, keep2, 4, mask8, budget, ws8, kv_len=c.kv_len)
            c2, acc2, pos2 = gv.alloc_cache8(p, cu8), torch.zeros_like(acc), torch.zeros_like(pos)
            gv.gvote_prune8(p, c, mask8, c2, ws8, acc=acc, acc_out=acc2, token_pos=pos, token_pos_out=pos2)
            for (r, h) in weights:
                n = weights[r, h].size
                a = acc[h, cu8[r]:cu8[r] + n].cpu().numpy()
                assert np.allclose(a, weights[r, h], rtol=1e-4, atol=1e-6)
                idx = np.flatnonzero(co.evict(a, int(keep2[r, h]), 4, 4))
                for w in range(2):
                    codes[w, r, h] = co.quantise(co.values(*codes[w, r, h])[idx])
                weights[r, h], where[r, h] = a[idx].astype(np.float64), where[r, h][idx]
            c, acc, pos = c2, acc2, pos2
        gv.gvote_append8(p, k_new.cuda(), v_new.cuda(), one, 1, c, c.kv_len, ws8, acc=acc, token_pos=pos,
                         pos_new=dev(np.array([300 + step, 41 + step], dtype=np.int32)))
        out, lse = torch.zeros(batch, hq, d, dtype=torch.bfloat16).cuda(), torch.zeros(batch, hq).cuda()
        gv.gvote_attend8(p, q_new.cuda(), one, 1, c, out, ws8, lse=lse, acc=acc, acc_out=acc)
        for (r, h) in weights:
            for w, X in enumerate((k_new, v_new)):
                codes[w, r, h] = co.append(*codes[w, r, h], X[h, r:r + 1].double().numpy())
            where[r, h] = np.append(where[r, h], (300, 41)[r] + step)
            n = where[r, h].size
            same(read_cache(gv, c, 0, r, h, n), codes[0, r, h])
            same(read_cache(gv, c, 1, r, h, n), codes[1, r, h])
            assert np.array_equal(pos[h, cu8[r]:cu8[r] + n].cpu().numpy(), where[r, h])
            q = q_new[r:r + 1, h * g:(h + 1) * g].double().numpy()
            before = np.append(weights[r, h], 0.0)
            got = acc[h, cu8[r]:cu8[r] + n].double().cpu().numpy()
            check_attend(q, co.values(*codes[0, r, h]), co.values(*codes[1, r, h]),
                         out[r:r + 1, h * g:(h + 1) * g].double().cpu().numpy(),
                         lse[r:r + 1, h * g:(h + 1) * g].double().cpu().numpy(), None, before, got)
            weights[r, h] = got                                     # carry the device's sums on
    assert gv.gvote_poll_status(ws) == 0 and gv.gvote_poll_status(ws8) == 0


@gpu
def test_gvotes_own_mask_feeds_the_cache(gv):
    """gvote_evict's mask in gvote_compact and gvote_pack, and their rows against gvote_store8's."""
    rng = np.random.default_rng(13)
    p, lens = params(gv, 4, 2, 64), (500, 77)
    cu, total = cumulative(lens), 577
    K, V = (bf16(rng, 2, total, 64) for _ in range(2))
    acc = dev(rng.random((2, total)).astype(np.float32))
    geom = (2, total, 500)
    ws8, ws = workspace(gv, p, geom), gv.alloc_workspace(p, *geom)
    mask = torch.zeros(2, gv.mask_row_words(total, 2), dtype=torch.int32).cuda()
    budget, b2 = (torch.zeros(2, 2, dtype=torch.int32).cuda() for _ in range(2))
    gv.gvote_evict(p, acc, dev(cu), geom, dev(np.array([[200, 90], [77, 1]], dtype=np.int32)), 16, mask, budget, ws8)
    a, b = gv.alloc_cache8(p, cu), gv.alloc_cache8(p, cu)
    gv.gvote_store8(p, K.cuda(), V.cuda(), dev(cu), geom, a, ws8, mask=mask)
    Kc, Vc = K.cuda(), V.cuda()
    gv.gvote_compact(p, Kc, Vc, mask, dev(cu), geom, b2, ws)
    assert torch.equal(budget, b2) and torch.equal(a.kv_len, budget)
    gv.gvote_store8(p, Kc, Vc, dev(cu), geom, b, ws8, kv_len=b2)
    for x, y in ((a.K, b.K), (a.V, b.V), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale), (a.kv_len, b.kv_len)):
        assert torch.equal(x, y)


@gpu
def test_python_face_refuses_other_shapes(gv):
    p = params(gv, 4, 2, 64)
    c = gv.alloc_cache8(p, [0, 100])
    ws = workspace(gv, p, c.geom, 1, 1)
    Q = torch.zeros(1, 4, 64, dtype=torch.bfloat16).cuda()
    cq = dev(cumulative((1,)))
    for bad in (dict(Q=Q.float()), dict(Q=Q[:, :3]), dict(out=Q[..., :32]), dict(cu_q=cq.long()), dict(lse=torch.zeros(1, 3).cuda()),
                dict(acc_out=torch.zeros(2, 99).cuda()), dict(ws=ws.cpu()), dict(cache=gv.alloc_cache8(params(gv, 4, 2, 32), [0, 100])),
                dict(max_q=0), dict(max_q=2)):
        a = {**dict(Q=Q, cu_q=cq, max_q=1, cache=c, out=Q.clone(), ws=ws), **bad}
        with pytest.raises((TypeError, ValueError, gv.GVoteError)):
            gv.gvote_attend8(p, **a)
    with pytest.raises(gv.GVoteError, match="workspace"):
        gv.gvote_attend8(p, Q, cq, 1, c, Q.clone(), ws[:512])


@gpu
def test_a_cache_keeps_its_tensors(gv):
    """The pointers are taken once, so that another tensor in a field would not be seen: it is refused."""
    c = gv.alloc_cache8(params(gv, 4, 2, 64), [0, 100])
    for name in ("K", "V", "k_scale", "v_scale", "cu_seqlens", "kv_len", "geom", "args"):
        with pytest.raises(AttributeError, match="fixed"):
            setattr(c, name, getattr(c, name))
