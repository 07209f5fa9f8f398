"""Numbers that name no page, in tables and on the stack: gvote_page_tables changes nothing and says so, in every form of the
call (one CTA and a cluster, pages kept by their threads and pages that go by way of the stack, more entries than a CTA holds)."""
import numpy as np
import pytest
import torch

from oracle import attend_oracle as ao
from tests.attend_util import cu_of, dev
from tests.test_pages import State

INVALID = -1
LOW, HIGH = -(1 << 31), (1 << 31) - 1

# requests, heads, rows of each, room of a table, spare pages, new tokens of each, under a mask
FORMS = {
    "step": (5, 3, 46, 6, 60, 3, False),
    "cut": (4, 2, 16 * 800, 801, 5, 0, False),               # 6400 pages back: more than a CTA's threads keep
    "mask": (3, 2, 200, 40, 500, 300, True),
    "prompt": (2, 3, 100, 500, 2100, 5000, False),
    "far": (8, 5, 16 * 900, 1000, 1000, 230, True),          # 36000 pages back: more than a cluster's threads keep
    "many": (600, 8, 31, 4, 5000, 2, False),
}


@pytest.fixture(scope="module")
def gv():
    from paper_2509_03136_b200 import gvote
    return gvote


def make(gv, form):
    B, H, rows, room, spare, new, masked = FORMS[form]
    s = State(gv, B, H, 16, np.full((B, H), rows), room, spare, seed=B)
    lens = [new] * B if new else None
    kept = np.random.default_rng(1).random((H, B * new)) < 0.9 if masked else None
    return s, np.zeros((B, H), int), lens, kept


def put(s, where, value):
    """One number of the tables or of the stack, on both sides; what it was."""
    host, there = (s.tabs, s.pages.tables) if len(where) == 3 else (s.free, s.pages.free)
    was = int(host[where])
    host[where] = value
    there[where] = int(value)
    return was


@pytest.mark.gpu
@pytest.mark.parametrize("form", list(FORMS))
def test_released_numbers(gv, form):
    s, keep, lens, kept = make(gv, form)
    B, H = s.kv.shape
    last = -(-int(s.kv[0, 0]) // 16) - 1
    n = s.pages.K.shape[0]
    for where, value in (((0, 0, 0), -1), ((B - 1, H - 1, last), n), ((B // 2, 0, last // 2), HIGH), ((B - 1, 0, 0), LOW)):
        was = put(s, where, value)
        assert s.step(keep, lens, kept) == INVALID
        put(s, where, was)
    put(s, (0, 0, last + 1), HIGH)                                    # behind the last page: not looked at
    assert s.step(keep, lens, kept) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("form", [f for f in FORMS if f not in ("cut", "far")])
def test_taken_numbers(gv, form):
    s, _, lens, kept = make(gv, form)
    P, n = 16, s.pages.K.shape[0]
    new = ao.tables(s.tabs, s.kv, s.free, s.n_free, P, None, cu_of(lens), kept)
    top, end = s.n_free, int(new[3])                                  # the stack's numbers end .. top - 1 are taken
    assert end < top - 1
    for where, value in ((top - 1, -1), (end, n), ((top + end) // 2, LOW)):
        was = put(s, (where,), value)
        assert s.step(None, lens, kept) == INVALID
        put(s, (where,), was)
    if end:
        put(s, (end - 1,), HIGH)                                      # stays on the stack
    assert s.step(None, lens, kept) == 0


@pytest.mark.gpu
def test_taken_numbers_below_many_released_ones(gv):
    """A few pages more than were released: the last ones come from the stack as it was."""
    s = State(gv, 6, 1, 16, np.full((6, 1), 16 * 900), 910, 90, seed=3)
    lens = [16 * 905] * 6
    was = put(s, (90 - 30,), -5)
    assert s.step(np.zeros((6, 1), int), lens) == INVALID
    put(s, (90 - 30,), was)
    assert s.step(np.zeros((6, 1), int), lens) == 0
    assert s.n_free == 60


@pytest.mark.gpu
@pytest.mark.parametrize("new,masked", [(3, False), (20, False), (5000, False), (700, True)])
def test_rows_that_go_on_in_no_page(gv, new, masked):
    """The page under a head's last rows does not exist: the rows that would go on in it have no place, the others theirs."""
    B, H, P = 2, 2, 16
    s = State(gv, B, H, P, np.full((B, H), 37), 700, 1500, seed=4)
    lens, n = [new] * B, s.pages.K.shape[0]
    kept = np.ones((H, B * new), bool) if masked else None
    want = ao.tables(s.tabs, s.kv, s.free, s.n_free, P, None, cu_of(lens), kept)
    for value in (-1, n):
        s = State(gv, B, H, P, np.full((B, H), 37), 700, 1500, seed=4)
        put(s, (1, 0, 2), value)
        slots = torch.zeros(H, B * new, dtype=torch.int32, device="cuda")
        mask = None
        if masked:
            from tests.test_pages import pack_mask
            mask = dev(pack_mask(kept, cu_of(lens)))
        gv.gvote_page_tables(s.p, s.pages, s.ws, cu_new=dev(cu_of(lens)), max_new=new, slots=slots, mask=mask)
        assert gv.gvote_poll_status(s.ws) == INVALID
        expect = want[4].copy()
        expect[0, new:new + min(new, 11)] = -1                        # 37 rows: eleven more to the end of the third page
        assert np.array_equal(slots.cpu().numpy(), expect)


def test_the_oracle_refuses_such_numbers():
    tabs, free = np.array([[[2, 7, 9]]], np.int32), np.array([0, 1, 5, 3], np.int32)
    kv = np.array([[32]], np.int32)
    assert ao.tables(tabs, kv, free, 2, 16, np.array([[0]])) is None               # 7 is none of four pages
    assert ao.tables(tabs, kv, free, 2, 16, np.array([[32]])) is not None
    ok = np.array([[[2, 1, 9]]], np.int32)
    assert ao.tables(ok, kv, free, 1, 16, np.array([[0]]), np.array([0, 33])) is not None
    assert ao.tables(ok, kv, free, 3, 16, None, np.array([0, 16])) is None         # 5 lies on top
