"""gvote_page_tables and gvote_page_write against plain loops: whole numbers and copies, so everything is equal."""
import numpy as np
import pytest
import torch

from oracle import attend_oracle as ao
from tests.attend_util import cu_of, dev, params

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gv():
    from paper_2509_03136_b200 import gvote
    return gvote


def pack_mask(kept, cu):
    """Bits [hkv, total] -> mask words, each request on a word of its own."""
    H, total = kept.shape
    words = np.zeros((H, (total >> 5) + len(cu) - 1), np.uint32)
    for r in range(len(cu) - 1):
        for t in range(cu[r], cu[r + 1]):
            i = t - cu[r]
            words[:, (cu[r] >> 5) + r + (i >> 5)] |= kept[:, t].astype(np.uint32) << np.uint32(i & 31)
    return words.view(np.int32)


class State:
    def __init__(self, gv, B, H, P, rows, max_pages, spare, seed=0, d=16):
        rng = np.random.default_rng(seed)
        self.gv, self.P, self.p = gv, P, params(gv, H, H, d)
        used = -(-rows // P)
        n = int(used.sum()) + spare
        order = rng.permutation(n).astype(np.int32)
        self.tabs = rng.integers(-5, n + 5, (B, H, max_pages)).astype(np.int32)   # behind the last page: anything
        at = 0
        for r in range(B):
            for h in range(H):
                k = used[r, h]
                self.tabs[r, h, :k] = order[at:at + k]
                at += k
        self.free = rng.integers(-9, -1, n).astype(np.int32)
        self.free[:spare] = order[at:]
        self.kv, self.n_free = rows.astype(np.int32), spare
        K = torch.zeros(n, P, d, dtype=torch.bfloat16, device="cuda")
        self.pages = gv.PageCache(K, torch.zeros_like(K), dev(self.tabs), dev(self.kv), dev(self.free), dev(np.array([spare], np.int32)))
        self.ws = gv.alloc_attend_workspace(self.p, B)

    def step(self, keep=None, lens=None, kept=None, lead=0, trail=0):
        """One call; the state is compared with the oracle's and becomes it.  Returns the slots, or None after a refusal."""
        gv, cu = self.gv, None
        if lens is not None:
            cu = cu_of(lens) + np.int32(lead)
        total = 0 if cu is None else int(cu[-1]) + trail
        H = self.tabs.shape[1]
        slots = None if cu is None else torch.full((H, total), 99, dtype=torch.int32, device="cuda")
        want = ao.tables(self.tabs, self.kv, self.free, self.n_free, self.P, keep, cu, kept)
        mask = None
        if kept is not None:
            padded = np.zeros((H, total), bool)
            padded[:, :kept.shape[1]] = kept
            mask = dev(pack_mask(padded, cu))
        gv.gvote_page_tables(self.p, self.pages, self.ws, keep=None if keep is None else dev(keep.astype(np.int32)),
                             cu_new=None if cu is None else dev(cu), max_new=0 if cu is None else max(lens), slots=slots, mask=mask)
        status = gv.gvote_poll_status(self.ws)
        gv.gvote_clear_status(self.ws)
        if want is None:
            assert status in (-1, -3)
            want = (self.tabs, self.kv, self.free, self.n_free, np.full((H, total), -1))
        else:
            assert status == 0
        now = [x.cpu().numpy() for x in (self.pages.tables, self.pages.kv_len, self.pages.free, self.pages.n_free)]
        assert np.array_equal(now[0], want[0]) and np.array_equal(now[1], want[1])
        assert np.array_equal(now[2], want[2]) and now[3][0] == want[3]
        if slots is not None:
            full = np.full((H, total), -1)
            full[:, :want[4].shape[1]] = want[4]
            assert np.array_equal(slots.cpu().numpy(), full)
        self.tabs, self.kv, self.free, self.n_free = now[0], now[1], now[2], int(now[3][0])
        return status


@pytest.mark.parametrize("B,H,P", [(1, 1, 16), (3, 2, 16), (130, 8, 16), (5, 4, 64), (2, 3, 1024)])
def test_a_life_of_steps(gv, B, H, P):
    rng = np.random.default_rng(B)
    rows = rng.integers(0, 3 * P, (B, H))
    rows[0, 0] = P                                                    # a page that is just full
    s = State(gv, B, H, P, rows, 9, B * H * 5 + 3, seed=B)
    for i in range(6):
        lens = rng.integers(0, 5 if i % 2 else P, B).tolist()
        keep = None if i == 1 else np.maximum(s.kv - rng.integers(-2, 2 * P if i == 4 else 4, (B, H)), -1)
        assert s.step(keep, lens, lead=i % 3, trail=i) == 0
    assert s.step(np.zeros((B, H), int)) == 0                         # every request ends
    assert s.n_free == s.pages.K.shape[0] and not s.kv.any()
    assert s.step() == 0                                              # nothing asked for


@pytest.mark.parametrize("lens", [[1], [5000, 0, 31, 32, 33], [9000, 4096, 4097], [700] * 20])
@pytest.mark.parametrize("H", [1, 3])
def test_masks(gv, lens, H):
    rng = np.random.default_rng(len(lens))
    total = sum(lens)
    kept = rng.random((H, total)) < rng.random((H, 1))
    cu = cu_of(lens)
    kept[0, cu[0]:cu[1]] = True
    if H > 1:
        kept[1, :] = False
    s = State(gv, len(lens), H, 16, rng.integers(0, 90, (len(lens), H)), 700, total * H // 16 + 3 * len(lens) * H, seed=1)
    assert s.step(None, lens, kept) == 0
    assert s.step(np.zeros((len(lens), H), int), lens, kept) == 0     # the same again in place of what it grew
    assert s.step(np.zeros((len(lens), H), int), lens, kept, lead=0, trail=40) == 0
    assert s.step(None, [40] * len(lens)) == 0


@pytest.mark.parametrize("lens", [[9000, 1], [3000] * 4])
def test_long_prompts_without_a_mask(gv, lens):
    s = State(gv, len(lens), 2, 16, np.full((len(lens), 2), 7), 700, 3000)
    assert s.step(None, lens, lead=5, trail=3) == 0


def test_cutting_what_was_grown_restores_the_stack(gv):
    s = State(gv, 40, 4, 16, np.random.default_rng(3).integers(0, 60, (40, 4)), 8, 500)
    stack, n, held = s.free[:s.n_free].copy(), s.n_free, s.kv.copy()
    assert s.step(None, [20] * 40) == 0
    assert s.step(held) == 0
    assert s.n_free == n and np.array_equal(s.free[:n], stack)


@pytest.mark.parametrize("H", [4, 5])
@pytest.mark.parametrize("first_rows", [15, 16, 17, 33])
@pytest.mark.parametrize("first_new", [0, 1, 17])
def test_a_thousand_pages_change_hands(gv, H, first_rows, first_new):
    """256 requests of 4 heads give back and take 1024 pages, a few more or less: all heads lose what they held and grow at once."""
    rows = np.full((256, H), 16)
    rows[0] = first_rows
    s = State(gv, 256, H, 16, rows, 4, 9, seed=first_rows)
    assert s.step(np.zeros((256, H), int), [first_new] + [1] * 255) == 0
    assert s.step(s.kv - 1, [2] * 256) in (0, -3)                     # (pages of one row: back and out again, one more where there was none)
    assert s.step(np.zeros((256, H), int), [1] * 255 + [0]) == 0


@pytest.mark.parametrize("long_ones", [False, True])
def test_refusals_change_nothing(gv, long_ones):
    n = 6000 if long_ones else 20
    s = State(gv, 3, 2, 16, np.full((3, 2), 16), 400, 5, seed=2)      # too few pages
    assert s.step(None, [n] * 3) == -3
    # (3 + 20 rows take one more page of each of four heads, and five are there)
    assert s.step(np.full((3, 2), 3), [n, 0, n], kept=np.ones((2, 2 * n), bool)) == (-3 if long_ones else 0)
    assert s.step(np.full((3, 2), 3)) == 0
    s = State(gv, 3, 2, 16, np.full((3, 2), 16), 2, 3000, seed=2)     # a table of two pages
    assert s.step(None, [16, 17, 16]) == -3
    assert s.step(None, [16, 16, 16]) == 0
    for bad in (-1, s.pages.K.shape[0] + 1):                          # not a height
        s.pages.n_free.fill_(bad)
        s.n_free = bad
        assert s.step(np.zeros((3, 2), int), [1, 1, 1]) == -1
    s.pages.n_free.fill_(s.pages.K.shape[0] - 2)                      # pages that would be on the stack twice
    s.n_free = s.pages.K.shape[0] - 2
    assert s.step(np.zeros((3, 2), int)) == -1


def test_lengths_out_of_range_are_clamped(gv):
    s = State(gv, 2, 2, 16, np.array([[20, 32], [0, 5]]), 2, 20, seed=5)
    s.pages.kv_len[0, 1], s.pages.kv_len[1, 0] = 1 << 30, -7
    s.kv[0, 1], s.kv[1, 0] = 1 << 30, -7
    assert s.step(np.array([[20, 30], [4, 4]]), [1, 2]) == 0


def test_repeats_in_a_graph(gv):
    s = State(gv, 4, 2, 16, np.full((4, 2), 30), 20, 200)
    cu, slots = dev(cu_of([1, 1, 0, 1])), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        gv.gvote_page_tables(s.p, s.pages, s.ws, cu_new=cu, max_new=1, slots=slots)
    for _ in range(40):
        want = ao.tables(s.tabs, s.kv, s.free, s.n_free, 16, None, cu_of([1, 1, 0, 1]))
        graph.replay()
        torch.cuda.synchronize()
        s.tabs, s.kv, s.free, s.n_free = want[:4]
        assert np.array_equal(slots.cpu().numpy(), want[4])
    assert np.array_equal(s.pages.tables.cpu().numpy(), s.tabs) and np.array_equal(s.pages.kv_len.cpu().numpy(), s.kv)


@pytest.mark.parametrize("d", [16, 64, 80, 128, 208, 256])
@pytest.mark.parametrize("split", [False, True])
def test_write(gv, d, split):
    g = torch.Generator().manual_seed(d)
    H, total, n, P = 3, 333, 90, 32
    p = params(gv, H, H, d)
    new = torch.randn(2, total, H, d + 8, generator=g).bfloat16()
    K_new, V_new = (x.cuda()[..., :d].transpose(0, 1) for x in new)
    order = torch.randperm(n * P, generator=g)[:H * total].view(H, total).int()
    order[torch.rand(H, total, generator=g) < 0.4] = -1
    order[0, 100:140] = -7
    order[2, :] = -1
    mem = torch.full((n, 2, P, d) if split else (2, n, P, d), 5.0).bfloat16()
    dev_mem = mem.cuda()
    view = lambda m: (m[:, 0], m[:, 1]) if split else (m[0], m[1])
    K, V = view(dev_mem)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    pages = gv.PageCache(K, V, i32(1, H, 4), i32(1, H), i32(n), i32(1))
    ws = gv.alloc_attend_workspace(p, 1)
    gv.gvote_page_write(p, K_new, V_new, order.cuda(), pages, ws)
    assert gv.gvote_poll_status(ws) == 0
    for want, rows, got in zip(view(mem), new, view(dev_mem)):
        for h in range(H):
            for t in (order[h] >= 0).nonzero()[:, 0].tolist():
                want[order[h, t] // P, order[h, t] % P] = rows[t, h, :d]
        assert torch.equal(got.cpu(), want)
    bad = order.clone()
    bad[1, 5] = n * P
    dev_mem.copy_(torch.full_like(mem, 5.0))
    gv.gvote_page_write(p, K_new, V_new, bad.cuda(), pages, ws)
    assert gv.gvote_poll_status(ws) == -1
    gv.gvote_clear_status(ws)
    if order[1, 5] >= 0:
        for want in view(mem):
            want[order[1, 5] // P, order[1, 5] % P] = 5.0
    assert torch.equal(dev_mem.cpu(), mem)                            # the others went to their places


def test_prompt_to_decode(gv):
    """A run as an engine makes it: prompts attended to, pruned, put into pages; drafts come, some are rejected; at every
    step the paged cache answers what plain rows do."""
    from tests.attend_util import Case, compare
    rng = np.random.default_rng(0)
    hq, H, d, P = 8, 2, 64, 16
    lens = [300, 77, 150]
    p = params(gv, hq, H, d)
    case = Case(hq, H, d, [[n] * H for n in lens], lens, seed=1)
    K, V, cu, _, geom = case.slabs(room=0)
    ws = gv.alloc_attend_workspace(p, 3, sum(lens), max(lens))
    wide, out, lse = case.outputs()
    gv.gvote_attend(p, case.Q.cuda(), cu, max(lens), K, V, cu, geom, out, ws, lse=lse)
    case.check(wide, out, lse, 2.0 ** -8)
    # evict by the weight the prompt's queries gave, heads keep different numbers of rows
    ws8 = gv.alloc_cache_workspace(p, *geom, sum(lens), max(lens))
    acc = torch.zeros(H, sum(lens), device="cuda")
    gv.gvote_accumulate(p, case.Q.cuda(), cu, max(lens), K, cu, geom, acc, ws8, lse=lse)
    keep = dev(rng.integers(20, 70, (3, H)).astype(np.int32))
    mask = torch.zeros(H, gv.mask_row_words(sum(lens), 3), dtype=torch.int32, device="cuda")
    budget = torch.zeros(3, H, dtype=torch.int32, device="cuda")
    gv.gvote_evict(p, acc, cu, geom, keep, 8, mask, budget, ws8)
    pages = gv.alloc_pages(p, 3, 80, P, 12)
    slots = torch.zeros(H, sum(lens), dtype=torch.int32, device="cuda")
    gv.gvote_page_tables(p, pages, ws, cu_new=cu, max_new=max(lens), slots=slots, mask=mask)
    gv.gvote_page_write(p, K, V, slots, pages, ws)
    assert torch.equal(pages.kv_len, budget)
    host_cu = cu.cpu().numpy()
    have = [[[], []] for _ in lens]                                   # rows per request and head: keys, values
    for r in range(3):
        for w, x in enumerate((case.K, case.V)):
            for h in range(H):
                bits = gv.unpack_mask(mask[h].cpu().numpy(), gv.mask_word_offset(int(host_cu[r]), r), lens[r])
                have[r][w].append(x[r][h][torch.from_numpy(bits)])
    accepted = None
    for n_new in (1, 4, 3, 40):
        if accepted is not None:
            for r in range(3):
                for w in range(2):
                    have[r][w] = [x[:accepted[r, h]] for h, x in enumerate(have[r][w])]
        step = Case(hq, H, d, [[n_new] * H] * 3, [n_new] * 3, seed=n_new)
        for r in range(3):
            for w, x in enumerate((step.K, step.V)):
                have[r][w] = [torch.cat([have[r][w][h], x[r][h]]) for h in range(H)]
        cu_new = dev(step.cu_q)
        slots = torch.zeros(H, 3 * n_new, dtype=torch.int32, device="cuda")
        gv.gvote_page_tables(p, pages, ws, keep=None if accepted is None else dev(accepted.astype(np.int32)), cu_new=cu_new,
                             max_new=n_new, slots=slots)
        rows = lambda x: torch.stack([torch.cat([x[r][h] for r in range(3)]) for h in range(H)]).cuda()
        gv.gvote_page_write(p, rows(step.K), rows(step.V), slots, pages, ws)
        wide, out, lse = step.outputs()
        gv.gvote_page_attend(p, step.Q.cuda(), cu_new, n_new, pages, out, ws, lse=lse)
        assert gv.gvote_poll_status(ws) == 0
        step.K, step.V = [h[0] for h in have], [h[1] for h in have]
        step.check(wide, out, lse, 2.0 ** -16 if n_new * hq // H <= 16 else 2.0 ** -8)
        held = np.array([[x.shape[0] for x in h[0]] for h in have])
        assert np.array_equal(pages.kv_len.cpu().numpy(), held)
        accepted = held - rng.integers(0, n_new, (3, 1))              # some drafts are rejected, of every head alike
    gv.gvote_page_tables(p, pages, ws, keep=torch.zeros(3, H, dtype=torch.int32, device="cuda"))
    assert int(pages.n_free) == 80 and sorted(pages.free.tolist()) == list(range(80))


def test_more_entries_than_a_thread_block_holds(gv):
    """Beyond 4096 (request, head) pairs the lengths are read for every phase."""
    rng = np.random.default_rng(7)
    s = State(gv, 700, 8, 16, rng.integers(0, 40, (700, 8)), 6, 700 * 8 * 2, seed=9)
    assert s.step(np.maximum(s.kv - rng.integers(0, 20, (700, 8)), 0), rng.integers(0, 3, 700).tolist()) == 0
    assert s.step(None, rng.integers(0, 20, 700).tolist()) == 0
    assert s.step(s.kv - 1, rng.integers(0, 2, 700).tolist(), lead=3, trail=2) == 0
    assert s.step(np.zeros((700, 8), int)) == 0
