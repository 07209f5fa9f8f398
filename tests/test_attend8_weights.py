"""gvote_attend8 where one row holds nearly all of the weight and the others carry the output: a weight is a 32-bit number,
however small it is beside the largest (a first row that collects the attention and has a small value is what a pruned cache
always keeps).  Bounds:
  logits    one product of stored values each (all other channels of the keys are zero): exact, but for the scaling,
            dl = 2^-22 |l|
  weights   relative 2 dl + 2^-20 (numerator and denominator; exponential, sum and log of a few units)
  out       half a step of bf16 (2^-8 |o|), then on sum w|v| the weight's error, and (n + 3) 2^-24 for the sums in 32 bits
            and the weight's own three terms
  lse       dl + 2^-20 + 2^-22 |lse|"""
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


def attend(gv, lens, hq, d, logits, V, n_q=1):
    """One KV head; `logits` [total] (values that e4m3 holds beside one another) times the query's first channel, which is
    about sqrt(d) 2^-j for query row j mod 3; V [total, d].  Returns the device's results and the oracle's inputs."""
    p = gv.make_params(d_h=64, n_q_heads=hq, n_kv_heads=1, d_k=d, rope_theta=1e4, S=8, p_nuc=0.95, n_f=1, n_s=4, seed=0)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    cq = np.arange(len(lens) + 1, dtype=np.int32) * n_q
    K = torch.zeros(1, int(cu[-1]), d)
    K[0, :, 0] = torch.from_numpy(logits.astype(np.float32))
    c = gv.alloc_cache8(p, cu)
    ws = gv.alloc_cache_workspace(p, *c.geom, int(cq[-1]), n_q)
    ws[256:].fill_(0xff)
    gv.gvote_store8(p, K.bfloat16().cuda(), torch.from_numpy(V.astype(np.float32)).bfloat16()[None].cuda(), c.cu_seqlens, c.geom, c, ws)
    Q = torch.zeros(int(cq[-1]), hq, d)
    Q[:, :, 0] = np.sqrt(d) * torch.pow(2.0, -(torch.arange(hq) % 3).float())
    Q = Q.bfloat16()
    out = torch.full((int(cq[-1]), hq, d), float("nan"), dtype=torch.bfloat16).cuda()
    lse = torch.full((int(cq[-1]), hq), float("nan")).cuda()
    gv.gvote_attend8(p, Q.cuda(), torch.from_numpy(cq).cuda(), n_q, c, out, ws, lse=lse)
    assert gv.gvote_poll_status(ws) == 0
    held = []
    for w, (codes, scale) in enumerate(((c.K, c.k_scale), (c.V, c.v_scale))):
        x = codes[0].view(torch.float8_e4m3fn).double().cpu().numpy()
        s = scale[0].double().cpu().numpy()
        rows = []
        for r, n in enumerate(lens):
            b = gv.cache8_block_offset(int(cu[r]), r)
            rows.append(co.values(x[cu[r]:cu[r + 1]], s[b:b + (n + 63) // 64]))
        held.append(rows)
    return out.double().cpu().numpy(), lse.double().cpu().numpy(), Q.double().numpy(), held


def check(lens, out, lse, Q, held, n_q=1):
    for r, n in enumerate(lens):
        t = slice(r * n_q, (r + 1) * n_q)
        k, v = held[0][r], held[1][r]
        o, l, _ = co.attend(Q[t], k, v)
        w, _ = co.softmax_rows(Q[t], k, n_q)
        logit = np.abs(np.einsum("igd,nd->ign", Q[t], k)).max() / np.sqrt(Q.shape[2])
        dl = 2.0 ** -22 * logit
        a = np.einsum("ign,nd->igd", w, np.abs(v))
        bound = 2.0 ** -8 * np.abs(o) + (2 * dl + 2.0 ** -20 + (n + 3) * 2.0 ** -24) * a
        off = np.abs(out[t] - o)
        assert (off <= bound).all(), (r, float((off / np.maximum(bound, 1e-300)).max()))
        assert (np.abs(lse[t] - l) <= dl + 2.0 ** -20 + 2.0 ** -22 * np.abs(l)).all()


def values(n, d, seed):
    """Rows of +-1 and 1, the first one zero: what the others hold is all of the output."""
    V = np.random.default_rng(seed).choice([-1.0, 1.0], size=(n, d))
    V[:, :d // 2] = 1.0
    V[0] = 0.0
    return V


@gpu
@pytest.mark.parametrize("gap", [16.0, 18.0, 24.0, 40.0, 72.0])
@pytest.mark.parametrize("lens,hq,d", [((2048,) * 150, 20, 64), ((700,) * 3, 4, 128), ((2048,), 8, 64), ((300, 64, 1), 12, 256),
                                       ((1000, 129), 24, 128), ((513,), 16, 80), ((40000,), 3, 64), ((900,), 40, 192)])
def test_rows_far_below_the_dominant_one_count(gv, gap, lens, hq, d):
    logits, V = [], []
    for r, n in enumerate(lens):
        x = np.full(n, -gap)
        x[0] = 0.0
        logits.append(x)
        V.append(values(n, d, r))
    args = attend(gv, lens, hq, d, np.concatenate(logits), np.concatenate(V))
    assert all(np.abs(args[0][r, :, 0]).min() > 0 for r, n in enumerate(lens) if n > 1)
    check(lens, *args)


@gpu
@pytest.mark.parametrize("at", [0, 70, 127, 128, 400])
def test_levels_of_weight_each_alone_in_a_channel(gv, at):
    """Rows 2^-14 apart, each with a channel to itself: every one of them is its channel's only output, at every place of the
    dominant row, before the others or behind them (the accumulated rows are then scaled down)."""
    n, d = 401, 64
    logits, V = np.full(n, -88.0), np.zeros((n, d))
    order = [at] + [i for i in range(7, n, 53) if i != at][:7]
    for j, i in enumerate(order):
        logits[i] = -8.0 * j
        V[i, j] = 1.0
    out, lse, Q, held = attend(gv, (n,), 6, d, logits, V)
    assert (out[0, :, :len(order)] > 0).all()
    check((n,), out, lse, Q, held)


@gpu
@pytest.mark.parametrize("n,hq,n_q", [(64, 4, 1), (60, 20, 1), (128, 8, 1), (64, 6, 4), (33, 24, 1)])
def test_every_term_of_a_weight_counts_where_the_outputs_cancel(gv, n, hq, n_q):
    """256 channels of random signs, of which many nearly cancel: there a weight that lacks its second term would show."""
    rng = np.random.default_rng(n + hq)
    logits = rng.choice(np.array([-8, -7.5, -7, -6.5, -6, -5.5, -5, -4.5, -4, -3.75, -3.25, -2.75, -2.25, -1.25, -0.5, 0]), size=n)
    args = attend(gv, (n,), hq, 256, logits, rng.choice([-1.0, 1.0], size=(n, 256)), n_q=n_q)
    check((n,), *args, n_q=n_q)


@gpu
def test_a_first_row_with_nearly_all_weight_and_a_small_value(gv):
    """As met in use: the first row holds 99.9 % of the weight, its value is a hundredth of the others'."""
    rng = np.random.default_rng(5)
    lens = (2000, 9000)
    logits, V = [], []
    for n in lens:
        x = np.round(rng.normal(size=n) * 2).clip(-4, 4) - 16
        x[0] = 0.0
        v = rng.normal(size=(n, 128))
        v[0] *= 0.01
        logits.append(x)
        V.append(v)
    check(lens, *attend(gv, lens, 7, 128, np.concatenate(logits), np.concatenate(V)))


@gpu
@pytest.mark.parametrize("hq,d", [(4, 64), (8, 128), (12, 128), (16, 256), (20, 64), (3, 192)])
@pytest.mark.parametrize("step", [46.0, 60.0, 80.0])
def test_a_reference_that_moves_late(gv, hq, d, step):
    """Every group of warps meets rows e^step above all it has seen, after several tiles: what it has summed up is scaled down by
    2^66 and more, and still is the only output of its channels."""
    n = 128 * 12 + 5
    logits, V = np.full(n, -step), np.zeros((n, d))
    logits[::3] = -step - 2
    V[:, :d // 2] = np.random.default_rng(hq).choice([-1.0, 1.0], size=(n, d // 2))
    V[:, 0] = 1.0
    for tile in range(8, 13):
        i = 128 * tile + tile % 5
        logits[i], V[i] = 0.0, 0.0
        V[i, d // 2:] = 1.0
    out, lse, Q, held = attend(gv, (n,), hq, d, logits, V)
    assert (out[0, :, 0] > 0).all()
    check((n,), out, lse, Q, held)


@gpu
@pytest.mark.parametrize("hq,d,n,batch", [(4, 64, 128 * 12, 150), (8, 128, 128 * 12, 150), (20, 64, 128 * 9, 150), (3, 192, 128 * 12, 150),
                                          (4, 64, 128 * 600, 1), (12, 80, 128 * 900, 1), (1, 64, 128 * 5000, 1)])
def test_three_levels_of_weight(gv, hq, d, n, batch):
    """Rows at e^-88, behind them rows at e^-48, behind them one at 1: the second level stays below the point at which what is summed
    up is scaled, and is then scaled by more than a float's exponents reach; across CTAs it is merged the same way.  (With 150
    requests a CTA has all of one, or most.)"""
    logits, V = np.full(n, -88.0), np.zeros((n, d))
    a, b = n // 3 // 128 * 128, 2 * n // 3 // 128 * 128
    logits[a:b] = -48.0
    logits[b:] = -80.0
    V[:, 3] = 1.0                                                    # (one value scale for all)
    V[a:b, 0], V[a:b, 1] = 1.0, np.random.default_rng(n).choice([-1.0, 1.0], size=b - a)
    if batch == 1:
        b = n - 128                                                  # only the last CTA meets the largest
    tail = np.arange(b + 5, n, 128)
    logits[tail] = 0.0
    V[tail, 2] = 1.0
    lens = (n,) * batch
    out, lse, Q, held = attend(gv, lens, hq, d, np.tile(logits, batch), np.tile(V, (batch, 1)))
    assert (out[:, :, 0] > 0).all()
    check(lens[:3], out, lse, Q, held)
    assert (out == out[0]).all() or np.allclose(out, out[0], rtol=2.0 ** -6, atol=0)
