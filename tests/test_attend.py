"""gvote_attend and gvote_page_attend against the definition in 64 bits: lengths, head layouts, strides, rows that see nothing,
and what lies in places that must not be read.

Weights enter the product with the values as two bf16 terms in calls of few query rows (rounded twice by at most 2^-8: 2^-16)
and as one bf16 in larger ones (2^-8)."""
import numpy as np
import pytest
import torch

from tests.attend_util import Case, compare, dev, params

pytestmark = pytest.mark.gpu
FEW, MANY = 2.0 ** -16, 2.0 ** -8


@pytest.fixture(scope="module")
def gv():
    from paper_2509_03136_b200 import gvote
    return gvote


def few(case):
    return max(case.nq) * (case.hq // case.hkv) <= 16 or case.d > 128


def run_pages(gv, case, page_rows, ws=None, head_pad=0, **kw):
    p = params(gv, case.hq, case.hkv, case.d)
    pages = case.pages(gv, page_rows, **kw)
    wide, out, lse = case.outputs(head_pad)
    ws = gv.alloc_attend_workspace(p, *case.geom()) if ws is None else ws
    gv.gvote_page_attend(p, case.Q.cuda(), dev(case.cu_q), case.geom()[2], pages, out, ws, lse=lse)
    assert gv.gvote_poll_status(ws) == 0
    return wide, out, lse


def run_slabs(gv, case, head_pad=0, ws=None, **kw):
    p = params(gv, case.hq, case.hkv, case.d)
    K, V, cu, kv, geom = case.slabs(**kw)
    wide, out, lse = case.outputs(head_pad)
    ws = gv.alloc_attend_workspace(p, *case.geom()) if ws is None else ws
    gv.gvote_attend(p, case.Q.cuda(), dev(case.cu_q), case.geom()[2], K, V, cu, geom, out, ws, lse=lse, kv_len=kv)
    assert gv.gvote_poll_status(ws) == 0
    return wide, out, lse


HEADS = [(8, 2, 64), (32, 8, 128), (7, 1, 128), (6, 3, 80), (5, 5, 96), (16, 1, 16), (24, 2, 48)]


@pytest.mark.parametrize("hq,hkv,d", HEADS + [(4, 2, 256), (8, 1, 192), (128, 1, 64), (40, 1, 144)])
@pytest.mark.parametrize("page", [16, 64])
def test_one_token(gv, hq, hkv, d, page):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 400]
    case = Case(hq, hkv, d, [[max(0, n - 7 * h) for h in range(hkv)] for n in lens], [1] * len(lens), seed=hq + d)
    w = FEW if few(case) else MANY
    case.check(*run_pages(gv, case, page), w)
    case.check(*run_slabs(gv, case), w)


@pytest.mark.parametrize("nq", [2, 5, 16, 32])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (4, 2, 128), (3, 1, 256), (6, 3, 80)])
def test_a_few_tokens(gv, nq, hq, hkv, d):
    lens = [nq + 3, nq, max(nq - 1, 1), 1, 64, 70, 200, 1000]         # some heads hold fewer rows than there are tokens
    case = Case(hq, hkv, d, [[n + 5 * h for h in range(hkv)] for n in lens], [nq, nq, nq, nq, 1, nq, 0, nq - 1], seed=nq)
    w = FEW if few(case) else MANY
    case.check(*run_pages(gv, case, 32), w)
    case.check(*run_slabs(gv, case), w)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (8, 2, 128), (28, 4, 128), (2, 2, 80), (128, 1, 16)])
@pytest.mark.parametrize("page", [16, 256])
def test_chunks_over_pages(gv, hq, hkv, d, page):
    nq = [65, 200, 129, 0, 33, 1]
    case = Case(hq, hkv, d, [[n + 40 * h + extra for h in range(hkv)] for n, extra in zip(nq, [0, 300, 128, 9, -20, 511])], nq, seed=d)
    case.check(*run_pages(gv, case, page), MANY)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (8, 2, 128), (7, 1, 128), (5, 5, 96), (48, 1, 32)])
@pytest.mark.parametrize("lens", [[1, 2, 127, 128, 129, 255, 300, 0, 66], [700], [65, 64, 63]])
def test_prompts(gv, hq, hkv, d, lens):
    case = Case(hq, hkv, d, [[n] * hkv for n in lens], lens, seed=len(lens))
    if few(case):
        pytest.skip("goes to the kernel for few rows")
    case.check(*run_slabs(gv, case, room=0), MANY)


def test_strides_and_rows_around(gv):
    """Interleaved pages, token-major slabs, padded rows; query tokens before the first and behind the last request stay."""
    for nq in ([1, 1], [3, 40], [130, 70]):
        case = Case(8, 2, 64, [[90, 151], [260, 200]], nq, lead=3, trail=2, seed=nq[0])
        w = FEW if few(case) else MANY
        case.check(*run_pages(gv, case, 16, split=True, head_pad=8), w)
        case.check(*run_slabs(gv, case, tokens_outer=True, width=8, head_pad=16), w)


@pytest.mark.parametrize("nq", [1, 4, 100])
def test_masked_places_may_hold_anything(gv, nq):
    """Non-finite keys and values: the tokens that see them get what the definition says, the others nothing of them."""
    case = Case(8, 2, 128, [[300, 170], [nq + 2, max(nq, 65)]], [nq, nq], seed=11)
    inf, nan = float("inf"), float("nan")
    for r, rr in enumerate(case.rows):
        for h, n in enumerate(rr):
            case.V[r][h][n - 1, 3] = nan                              # the last row: seen by the last token only
            case.V[r][h][n - 1, 5] = inf
            case.V[r][h][max(n - nq // 2 - 1, 0), 9] = -inf
    case.V[0][0][20, 7] = inf                                         # a row everyone sees
    case.V[0][1][n - 1 - 2 * nq if n > 2 * nq else 0, 8] = -inf
    w = FEW if few(case) else MANY
    case.check(*run_pages(gv, case, 16), w)
    case.check(*run_slabs(gv, case), w)
    case.K[1][0][case.rows[1][0] - 1, 0] = nan                        # a key that only the last token sees
    case.check(*run_pages(gv, case, 16), w)
    case.check(*run_slabs(gv, case), w)


@pytest.mark.parametrize("nq", [1, 90])
def test_extreme_logits(gv, nq):
    """Logits that grow along the rows by far more than a reference may be passed by, shrink, or are all alike."""
    for trend in ("up", "down", "flat"):
        case = Case(4, 1, 64, [[777], [nq]], [nq, nq], seed=5, outliers=False)
        for r in range(2):
            n = case.rows[r][0]
            t = torch.linspace(-60, 60, n) if n > 1 else torch.zeros(n)
            ramp = dict(up=t, down=-t, flat=0 * t)[trend]
            case.K[r][0][:] = 0
            case.K[r][0][:, 0] = ramp.bfloat16()
        case.Q[:] = 0
        case.Q[:, :, 0] = 8.0
        w = FEW if few(case) else MANY
        case.check(*run_pages(gv, case, 64), w)
        case.check(*run_slabs(gv, case), w)


@pytest.mark.parametrize("n_q", [1, 8, 128])
def test_long_rows_are_split_and_joined(gv, n_q):
    """Few rows of queries over a long axis; twice the same, to the bit; a workspace that has served other calls."""
    case = Case(8, 2, 128, [[20000, 333]], [n_q], seed=3)
    p = params(gv, 8, 2, 128)
    ws = gv.alloc_attend_workspace(p, 40, 4000, 400)
    other = Case(8, 2, 128, [[50, 400]] * 40, [1] * 40, seed=4)
    first = run_pages(gv, case, 64, ws=ws)
    case.check(*first, FEW if few(case) else MANY)
    other.check(*run_pages(gv, other, 16, ws=ws), FEW)
    again = run_pages(gv, case, 64, ws=ws)
    assert torch.equal(first[1], again[1]) and torch.equal(first[2], again[2])
    slabs = run_slabs(gv, case, ws=ws)
    assert torch.equal(first[1], slabs[1]) and torch.equal(first[2], slabs[2])


def test_many_requests(gv):
    """More (request, head) pairs than a launch takes; requests without rows or without tokens."""
    B = 700
    rng = np.random.default_rng(0)
    rows = rng.integers(0, 40, (B, 2)).tolist()
    nq = rng.integers(0, 2, B).tolist()
    case = Case(4, 2, 64, rows, nq, seed=8)
    case.check(*run_pages(gv, case, 16), FEW)
    nq = rng.integers(0, 60, B).tolist()
    case = Case(4, 2, 64, rows, nq, seed=9)
    case.check(*run_pages(gv, case, 16), MANY)


def test_nothing_to_do(gv):
    p = params(gv, 8, 2, 64)
    ws = gv.alloc_attend_workspace(p, 2, 4, 4)
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    cu = dev(np.zeros(3, np.int32))
    gv.gvote_attend(p, z(0, 8, 64), cu, 0, z(2, 0, 64), z(2, 0, 64), cu, (2, 0, 0), z(0, 8, 64), ws)
    out, lse = torch.full((4, 8, 64), 7.0, device="cuda").bfloat16(), torch.full((4, 8), 7.0, device="cuda")
    for max_q in (1, 4):                                              # tokens without any rows
        cu_q = dev(np.array([0, min(max_q, 3), 4], np.int32))
        cu_q[1] = 4 - max_q if max_q == 4 else 1
        n = 4 if max_q == 4 else 2
        cu_q[2] = n
        gv.gvote_attend(p, z(n, 8, 64), cu_q, max_q, z(2, 0, 64), z(2, 0, 64), cu, (2, 0, 0), out[:n], ws, lse=lse[:n])
        assert bool((out[:n] == 0).all()) and bool(torch.isneginf(lse[:n]).all())
    assert bool((out == 0).all())


def test_too_many_tokens_and_missing_pages_are_reported(gv):
    for nq, most in ((3, 2), (200, 100)):
        case = Case(8, 2, 64, [[300, 250]], [nq], seed=1)
        p = params(gv, 8, 2, 64)
        ws = gv.alloc_attend_workspace(p, 1, nq, nq)
        wide, out, lse = case.outputs()
        pages = case.pages(gv, 16)
        gv.gvote_page_attend(p, case.Q.cuda(), dev(case.cu_q), most, pages, out, ws, lse=lse)
        assert gv.gvote_poll_status(ws) == -1
        gv.gvote_clear_status(ws)
        pages.tables[0, 1, 3] = pages.K.shape[0]
        gv.gvote_page_attend(p, case.Q.cuda(), dev(case.cu_q), nq, pages, out, ws, lse=lse)
        assert gv.gvote_poll_status(ws) == -1
        gv.gvote_clear_status(ws)


def test_lse_is_optional_and_what_accumulate_takes(gv):
    """A prompt's attention leaves the lse that gvote_accumulate computes otherwise."""
    case = Case(8, 2, 64, [[200, 200], [77, 77]], [200, 77], seed=2)
    p = params(gv, 8, 2, 64)
    K, V, cu, _, geom = case.slabs(room=0)
    ws = gv.alloc_attend_workspace(p, *case.geom())
    wide, out, lse = case.outputs()
    gv.gvote_attend(p, case.Q.cuda(), cu, 200, K, V, cu, geom, out, ws)
    plain = out.clone()
    gv.gvote_attend(p, case.Q.cuda(), cu, 200, K, V, cu, geom, out, ws, lse=lse)
    assert torch.equal(plain, out)
    ws8 = gv.alloc_cache_workspace(p, *geom, 277, 200)
    a, b = torch.zeros(2, 277, device="cuda"), torch.zeros(2, 277, device="cuda")
    gv.gvote_accumulate(p, case.Q.cuda(), cu, 200, K, cu, geom, a, ws8)
    gv.gvote_accumulate(p, case.Q.cuda(), cu, 200, K, cu, geom, b, ws8, lse=lse)
    # both are sums of exp(l - lse) over up to 800 rows in 32 bits, lse off by at most 2^-15 either way at these sizes
    assert float(((a - b).abs() / a.abs().clamp_min(1e-3)).max()) < 2.0 ** -13


@pytest.mark.parametrize("nq", [1, 70])
def test_streams_and_graphs(gv, nq):
    case = Case(8, 2, 64, [[500, 450], [90, 200]], [nq, nq], seed=6)
    p = params(gv, 8, 2, 64)
    want = run_pages(gv, case, 16)
    pages, Q, cu = case.pages(gv, 16), case.Q.cuda(), dev(case.cu_q)
    wide, out, lse = case.outputs()
    ws = gv.alloc_attend_workspace(p, *case.geom())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        gv.gvote_page_attend(p, Q, cu, nq, pages, out, ws, lse=lse)
    side.synchronize()
    assert torch.equal(out, want[1]) and torch.equal(lse, want[2])
    graph = torch.cuda.CUDAGraph()
    out.fill_(7), lse.fill_(7)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        gv.gvote_page_attend(p, Q, cu, nq, pages, out, ws, lse=lse)
    for _ in range(3):
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[1]) and torch.equal(lse, want[2])
    pages.kv_len.sub_(20)                                              # the captured call reads the lengths as they are
    short = Case(8, 2, 64, [[480, 430], [70, 180]], [nq, nq], seed=6)
    for r in range(2):
        for h in range(2):
            short.K[r][h], short.V[r][h] = case.K[r][h][:short.rows[r][h]], case.V[r][h][:short.rows[r][h]]
    short.Q = case.Q
    graph.replay()
    torch.cuda.synchronize()
    short.check(wide, out, lse, FEW if few(case) else MANY)


@pytest.mark.parametrize("over_pages", [False, True])
def test_ragged_prompts(gv, over_pages):
    """More units than SMs, requests of very different length and empty ones among them."""
    rng = np.random.default_rng(4)
    lens = [0, 1200, 3, 64, 700, 0, 1, 129, 400, 256]
    case = Case(64, 4, 32, [[n + int(rng.integers(0, 90)) * h for h in range(4)] for n in lens], lens, seed=12)
    case.check(*(run_pages(gv, case, 32) if over_pages else run_slabs(gv, case)), MANY)


@pytest.mark.parametrize("hq,hkv,d,nq", [(8, 2, 64, 5), (16, 2, 128, 3), (28, 4, 128, 40), (4, 4, 96, 300), (64, 1, 64, 1)])
def test_cut_lists(gv, hq, hkv, d, nq):
    """Few query tiles over long rows: pieces of units on different SMs, joined; heads of very different length; a request that
    begins behind token 0 and others without tokens."""
    case = Case(hq, hkv, d, [[9000 - 2500 * (h % 3) for h in range(hkv)], [40] * hkv, [1500 + h for h in range(hkv)]], [nq, 0, nq], lead=2, seed=d)
    w = FEW if few(case) else MANY
    first = run_pages(gv, case, 64)
    case.check(*first, w)
    case.check(*run_slabs(gv, case), w)
    again = run_pages(gv, case, 64)
    assert torch.equal(first[1], again[1]) and torch.equal(first[2], again[2])


def test_one_request_behind_token_0(gv):
    for nq in (1, 90):
        case = Case(8, 2, 64, [[3000, 200]], [nq], lead=5, trail=1, seed=nq)
        w = FEW if few(case) else MANY
        case.check(*run_pages(gv, case, 32), w)
        case.check(*run_slabs(gv, case), w)


def test_not_finite_values_in_cut_lists(gv):
    case = Case(8, 2, 64, [[6000, 5000]], [20], seed=21)
    for h, n in enumerate(case.rows[0]):
        case.V[0][h][100, 3] = float("inf")
        case.V[0][h][n - 3, 4] = float("nan")
        case.V[0][h][n - 10, 5] = -float("inf")
        case.V[0][h][2000, 5] = float("inf")
    case.check(*run_pages(gv, case, 16), MANY)
    case.check(*run_slabs(gv, case), MANY)


@pytest.mark.parametrize("nq", [1, 30])
def test_values_that_are_no_numbers_in_queries_and_keys(gv, nq):
    """A query row that holds a NaN spoils itself alone; a key whose logit is +inf the tokens that see it."""
    case = Case(8, 2, 64, [[200, 90], [150, nq + 1]], [nq, nq], seed=31)
    case.Q[nq // 2, 3, 5] = float("nan")
    case.K[1][0][149, 0] = float("inf")
    case.Q[nq:, :, 0] = case.Q[nq:, :, 0].abs() + 0.5                 # +inf, not -inf
    w = FEW if few(case) else MANY
    case.check(*run_pages(gv, case, 16), w)
    case.check(*run_slabs(gv, case), w)


@pytest.mark.parametrize("hq,hkv,d,nq", [(100, 1, 64, 3), (65, 1, 128, 2), (33, 1, 32, 9), (3, 3, 112, 7)])
def test_groups_that_leave_a_tile_rows(gv, hq, hkv, d, nq):
    case = Case(hq, hkv, d, [[140 + 9 * h for h in range(hkv)], [nq] * hkv], [nq, nq], seed=hq)
    w = FEW if few(case) else MANY
    case.check(*run_pages(gv, case, 16), w)
    case.check(*run_slabs(gv, case), w)


@pytest.mark.parametrize("nq", [1, 100])
def test_offsets_past_32_bits(gv, nq):
    """Pages and slabs that lie behind the first 2^31 elements."""
    case = Case(8, 2, 64, [[300, 170]], [nq], seed=41)
    p = params(gv, 8, 2, 64)
    want = run_pages(gv, case, 64)
    small = case.pages(gv, 64)
    far = (1 << 31) // (64 * 64) + 1                                  # pages of 64 rows x 64 channels
    n = small.K.shape[0]
    pool = torch.empty(2, far + n, 64, 64, dtype=torch.bfloat16, device="cuda")
    pool[:, far:] = torch.stack([small.K, small.V])
    pages = gv.PageCache(pool[0], pool[1], (small.tables + far).clamp_max(far + n), small.kv_len,
                         torch.zeros(far + n, dtype=torch.int32, device="cuda"), small.n_free)
    ws = gv.alloc_attend_workspace(p, *case.geom())
    wide, out, lse = case.outputs()
    gv.gvote_page_attend(p, case.Q.cuda(), dev(case.cu_q), nq, pages, out, ws, lse=lse)
    assert gv.gvote_poll_status(ws) == 0 and torch.equal(out, want[1]) and torch.equal(lse, want[2])
    # new rows to the last page, by the slot map
    slots = torch.tensor([[(far + n - 1) * 64 + 63], [-1]], dtype=torch.int32, device="cuda")
    new = torch.full((2, 1, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    before = pool[:, far:].clone()
    gv.gvote_page_write(p, new, -new, slots, pages, ws)
    before[0, n - 1, 63], before[1, n - 1, 63] = 3.0, -3.0
    assert torch.equal(pool[:, far:].nan_to_num(7.0), before.nan_to_num(7.0))
    # slabs: the second head 2^31 elements behind the first
    K, V, cu, kv, geom = case.slabs()
    flat = pool.view(-1)
    stride = far * 64 * 64
    slab = [flat.as_strided((2, geom[1], 64), (stride, 64, 1), at) for at in (0, geom[1] * 64)]
    slab[0].copy_(K), slab[1].copy_(V)
    wide, out, lse = case.outputs()
    gv.gvote_attend(p, case.Q.cuda(), dev(case.cu_q), nq, *slab, cu, geom, out, ws, lse=lse, kv_len=kv)
    assert gv.gvote_poll_status(ws) == 0 and torch.equal(out, want[1]) and torch.equal(lse, want[2])


def test_requests_that_share_pages(gv):
    """Two requests with the same prefix: their tables name the same pages."""
    case = Case(8, 2, 64, [[128, 128]], [2], seed=51)
    p = params(gv, 8, 2, 64)
    pages = case.pages(gv, 16)
    both = gv.PageCache(pages.K, pages.V, pages.tables.repeat(2, 1, 1).contiguous(), pages.kv_len.repeat(2, 1).contiguous(), pages.free, pages.n_free)
    ws = gv.alloc_attend_workspace(p, 2, 4, 2)
    Q = case.Q.cuda().repeat(2, 1, 1)
    out, lse = torch.zeros(4, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 8, device="cuda")
    gv.gvote_page_attend(p, Q, dev(np.array([0, 2, 4], np.int32)), 2, both, out, ws, lse=lse)
    wide, one, one_lse = run_pages(gv, case, 16)
    assert torch.equal(out[:2], one) and torch.equal(out[2:], one) and torch.equal(lse[2:], one_lse)


def test_two_streams_with_workspaces_of_their_own(gv):
    cases = [Case(8, 2, 128, [[4000, 3000]], [n], seed=60 + n) for n in (1, 200)]
    p = params(gv, 8, 2, 128)
    want = [run_pages(gv, c, 32) for c in cases]
    held = [(c.pages(gv, 32), c.Q.cuda(), dev(c.cu_q), gv.alloc_attend_workspace(p, *c.geom()), torch.cuda.Stream()) for c in cases]
    outs = [c.outputs() for c in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, (pages, Q, cu, ws, stream), (_, out, lse) in zip(cases, held, outs):
            with torch.cuda.stream(stream):
                gv.gvote_page_attend(p, Q, cu, c.nq[0], pages, out, ws, lse=lse)
    torch.cuda.synchronize()
    for w, (_, out, lse) in zip(want, outs):
        assert torch.equal(w[1], out) and torch.equal(w[2], lse)


@pytest.mark.parametrize("nq", [1, 64])
def test_infinities_in_a_long_cache(gv, nq):
    """Rows that every token sees and that hold infinities: found without a walk over the cache for every output."""
    case = Case(4, 2, 128, [[24000, 900]], [nq], seed=71)
    case.V[0][0][5, 7] = float("inf")
    case.V[0][0][20001, 7] = -float("inf")
    case.V[0][0][20001, 100] = float("inf")
    case.V[0][1][899, 0] = float("nan")
    p = params(gv, 4, 2, 128)
    pages, Q, cu = case.pages(gv, 32), case.Q.cuda(), dev(case.cu_q)
    wide, out, lse = case.outputs()
    ws = gv.alloc_attend_workspace(p, *case.geom())
    gv.gvote_page_attend(p, Q, cu, nq, pages, out, ws, lse=lse)
    assert gv.gvote_poll_status(ws) == 0
    case.check(wide, out, lse, FEW if few(case) else MANY)
