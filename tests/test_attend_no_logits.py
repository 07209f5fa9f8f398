"""Keys whose logits are -inf: a token that sees no others gets out = 0 and lse = -inf whatever the values hold; other tokens
get what the definition says, and the values of such rows that are not finite.  On a few tokens and on many, in whole units
and in cut lists.

Tolerances are the oracle's: weights enter the product with the values as two bf16 terms in calls of few query rows (2^-16) and
as one in larger ones (2^-8)."""
import numpy as np
import pytest
import torch

from tests.attend_util import Case
from tests.test_attend import FEW, MANY, few, run_pages, run_slabs

gpu = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def gv():
    from paper_2509_03136_b200 import gvote
    return gvote


def lower(case, r, h, rows):
    """The logits of these rows become -inf for every query (of any other row nothing changes but channel 0)."""
    case.K[r][h][rows, 0] = -INF


def make(hq, hkv, d, rows, nq, seed):
    case = Case(hq, hkv, d, rows, nq, seed=seed)
    case.Q[:, :, 0] = case.Q[:, :, 0].abs() + 0.5                     # -inf times a positive number: no NaN
    return case


def check(gv, case, page=16):
    w = FEW if few(case) else MANY
    case.check(*run_pages(gv, case, page), w)
    case.check(*run_slabs(gv, case), w)


@gpu
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (5, 1, 128), (2, 2, 80)])
@pytest.mark.parametrize("nq", [4, 100])
def test_tokens_that_see_only_such_keys(gv, hq, hkv, d, nq):
    """Of a prompt the first rows: the first tokens see nothing else, the others of their warp do."""
    case = make(hq, hkv, d, [[nq] * hkv, [nq] * hkv], [nq, nq], seed=nq + d)
    first = nq // 2
    for h in range(hkv):
        lower(case, 0, h, slice(0, first))
        case.V[0][h][0, 3] = INF
        case.V[0][h][first - 1, 5] = NAN
        case.V[0][h][first - 1, 6] = -INF
    check(gv, case)


@gpu
@pytest.mark.parametrize("hq,hkv,d,nq", [(8, 2, 64, 1), (8, 2, 128, 4), (4, 1, 256, 2), (8, 2, 128, 40), (7, 1, 64, 30)])
def test_rows_that_all_tokens_see(gv, hq, hkv, d, nq):
    """One head whose keys are all such, one that has others; infinities in rows that all tokens see and in the last ones."""
    case = make(hq, hkv, d, [[300 + 11 * h for h in range(hkv)], [nq + 70] * hkv], [nq, nq], seed=nq)
    lower(case, 0, 0, slice(0, None))
    lower(case, 1, hkv - 1, slice(0, 64))
    for r, h in ((0, 0), (1, hkv - 1)):
        n = case.rows[r][h]
        case.V[r][h][10, 2] = INF
        case.V[r][h][11, 9] = NAN
        case.V[r][h][n - 1, 4] = -INF
        case.V[r][h][max(n - nq, 0), 7] = NAN
    check(gv, case)


@gpu
@pytest.mark.parametrize("hq,hkv,d,nq", [(8, 2, 64, 1), (8, 2, 128, 20), (4, 2, 64, 70)])
def test_cut_lists(gv, hq, hkv, d, nq):
    """Pieces whose logits are all -inf beside others that are not, and a head of nothing else: the same as uncut."""
    case = make(hq, hkv, d, [[9000, 7000]], [nq], seed=nq)
    lower(case, 0, 0, slice(0, 5000))
    lower(case, 0, 1, slice(0, None))
    for h in range(2):
        case.V[0][h][100, 3] = INF
        case.V[0][h][4000, 4] = NAN
        case.V[0][h][4001, 5] = -INF
        case.V[0][h][case.rows[0][h] - 1, 6] = INF
    check(gv, case, page=64)


def test_the_oracle_on_such_rows():
    """(Its own check, by hand: two rows, one of them without weight.)"""
    from oracle import attend_oracle as ao
    q = np.ones((2, 1, 2))
    k, v = np.array([[-np.inf, 0.0], [1.0, 1.0]]), np.array([[1.0, np.inf], [3.0, 4.0]])
    out, lse, _, _ = ao.attend(q, k, v, 0.0)
    assert np.array_equal(out[0, 0], [0.0, 0.0]) and np.isneginf(lse[0, 0])
    assert np.array_equal(out[1, 0], [3.0, np.inf]) and lse[1, 0] == pytest.approx(2 / np.sqrt(2))
