"""gvote_page_write where rows have the same slot, which a caller is not to ask for: the place holds 16-byte pieces of any of these
rows, and every other place what it should."""
import pytest
import torch

from tests.attend_util import params


@pytest.mark.gpu
@pytest.mark.parametrize("d", [16, 80, 128, 256])
@pytest.mark.parametrize("apart", [1, 9, 200])
def test_pieces_are_of_one_of_the_rows(d, apart):
    from paper_2509_03136_b200 import gvote as gv
    H, total, n, P = 2, 400, 60, 16
    p = params(gv, H, H, d)
    g = torch.Generator().manual_seed(d + apart)
    new = torch.randn(2, H, total, d, generator=g).bfloat16()
    slots = torch.randperm(n * P, generator=g)[:H * total].view(H, total).int()
    twice = [(0, 3), (0, 40), (1, 100)]
    for h, t in twice:
        slots[h, t + apart] = slots[h, t]                             # of one warp's rows, of two warps', of two CTAs'
    slots[1, 399] = slots[0, 399]                                     # of two heads
    want = torch.full((2, n * P, d), 5.0).bfloat16()
    for h in range(H):
        want[:, slots[h].long()] = new[:, h]
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    K, V = (torch.full((n, P, d), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pages = gv.PageCache(K, V, i32(1, H, 4), i32(1, H), i32(n), i32(1))
    ws = gv.alloc_attend_workspace(p, 1)
    gv.gvote_page_write(p, new[0].cuda(), new[1].cuda(), slots.cuda(), pages, ws)
    assert gv.gvote_poll_status(ws) == 0
    got = torch.stack([K, V]).view(2, n * P, d).cpu()
    for rows in [[(h, t), (h, t + apart)] for h, t in twice] + [[(0, 399), (1, 399)]]:
        at = int(slots[rows[0]])
        piece = got[:, at].reshape(2, d // 8, 1, 8)
        from_rows = torch.stack([new[:, h, t] for h, t in rows], dim=2).view(2, d // 8, 8, len(rows)).transpose(2, 3)
        assert bool((piece == from_rows).all(dim=3).any(dim=2).all())
        want[:, at] = got[:, at] = 0
    assert torch.equal(got, want)
