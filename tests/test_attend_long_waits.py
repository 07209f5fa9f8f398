"""A unit of the many-row kernel that takes longer than its waits have tries for: they last as long as work is done."""
import math

import pytest
import torch

from tests.attend_util import dev, params

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1 << 20, 1 << 28])
def test_one_long_request_among_many(rows):
    """300 requests of one token and 17 query heads are more units than a cut list takes, so that one CTA walks over all rows of the
    long one (2^28: two seconds, as long as the waits' 2^20 tries).  Keys and values are the same memory: zeros, and ones in every
    1024th row.  The queries are zero, so the outputs are 2^-10 and lse the logarithm of the number of rows.

    Tolerances: weights are 2^0 within 2.1e-7, and a tile's 128 of them meet a sum that is a multiple of what 32 bits resolve
    there, as 128 is, so that a sum is within 4.2e-7 of rows; exponentials and sums together 2^-18, the logarithm four roundings.
    The products add whole numbers up to 2^18 (exact); the output is rounded to bf16 (2^-8)."""
    from paper_2509_03136_b200 import gvote as gv
    B, long_one, hq, d = 300, 150, 17, 16
    if torch.cuda.get_device_properties(0).total_memory < 4 * rows * d * 2:
        pytest.skip("not enough memory")
    p = params(gv, hq, 1, d)
    lens = [1] * B
    lens[long_one] = rows
    cu = torch.zeros(B + 1, dtype=torch.int64)
    cu[1:] = torch.tensor(lens).cumsum(0)
    total = int(cu[-1])
    x = torch.zeros(1, total, d, dtype=torch.bfloat16, device="cuda")
    x[0, long_one + 5:long_one + rows:1024] = 1.0
    Q = torch.zeros(B, hq, d, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(Q, 7.0), torch.full((B, hq), 7.0, device="cuda")
    ws = gv.alloc_attend_workspace(p, B, B, 1)
    gv.gvote_attend(p, Q, dev(range(B + 1)).int(), 1, x, x, cu.int().cuda(), (B, total, rows), out, ws, lse=lse)
    assert gv.gvote_poll_status(ws) == 0
    want, want_lse = torch.zeros(B, dtype=torch.float64), torch.zeros(B, dtype=torch.float64)
    want[long_one], want_lse[long_one] = 2.0 ** -10, math.log(rows)
    assert bool(((out.double().cpu() - want[:, None, None]).abs() <= 2.0 ** -8 * want[:, None, None]).all())
    tol = 2.0 ** -18 + 4 * 2.0 ** -24 * want_lse
    assert bool(((lse.double().cpu() - want_lse[:, None]).abs() <= tol[:, None]).all())
