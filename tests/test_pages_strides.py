"""K and V are laid out alike where their strides agree in all dimensions of more than one: a decode step of one request has
K_new [heads, 1, d] dense behind a rotation and V_new as a view of the projection's output."""
from types import SimpleNamespace

import pytest
import torch

from tests.attend_util import dev, params


@pytest.fixture(scope="module")
def gv():
    from paper_2509_03136_b200 import build
    build.build()
    from paper_2509_03136_b200 import gvote
    return gvote


def dense_and_view(H, n, d, device="cpu"):
    """Two tensors [H, n, d] of which the second is token-major with other channels behind."""
    return torch.randn(H, n, d, device=device).bfloat16(), torch.randn(n, H * d + 64, device=device).bfloat16()[:, :H * d].view(n, H, d).transpose(0, 1)


def calls(gv, device):
    """For a number of heads and of tokens: what takes K and V of these strides."""
    pages = SimpleNamespace(device=torch.device(device))
    slots, cu, ws = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(9, dtype=torch.uint8)
    def write(K, V):
        gv.gvote_page_write(params(gv, K.shape[0], K.shape[0], 64), K, V, slots, pages, ws)
    def slabs(K, V):
        gv.gvote_attend(params(gv, K.shape[0], K.shape[0], 64), torch.zeros(1, K.shape[0], 64).bfloat16(), cu, 1, K, V, cu, (1, K.shape[1], 1), None, ws)
    def cache(K, V):
        gv.PageCache(K, V, torch.zeros(1, 2, 3, dtype=torch.int32), cu, cu, cu)
    return write, slabs, cache


@pytest.mark.parametrize("which", [0, 1, 2])
def test_dimensions_of_one_may_have_any_stride(gv, which):
    call = calls(gv, "cpu")[which]
    with pytest.raises(TypeError, match="CUDA"):                      # (past the check of strides: refused for the device)
        call(*dense_and_view(8, 1, 64))
    with pytest.raises(TypeError, match="CUDA"):
        call(torch.zeros(1, 5, 64).bfloat16(), torch.zeros(2, 5, 64).bfloat16().as_strided((1, 5, 64), (640, 64, 1)))
    for n in (2, 5):
        with pytest.raises(ValueError, match="strides"):
            call(*dense_and_view(8, n, 64))


@pytest.mark.gpu
def test_one_token_in_two_layouts(gv):
    H, d, P = 8, 64, 16
    p = params(gv, 2 * H, H, d)
    K_new, V_new = dense_and_view(H, 1, d, "cuda")
    pages = gv.alloc_pages(p, 1, H, P, 2)
    ws = gv.alloc_attend_workspace(p, 1, 1, 1)
    slots = torch.zeros(H, 1, dtype=torch.int32, device="cuda")
    gv.gvote_page_tables(p, pages, ws, cu_new=dev([0, 1]).int(), max_new=1, slots=slots)
    gv.gvote_page_write(p, K_new, V_new, slots, pages, ws)
    assert gv.gvote_poll_status(ws) == 0
    at = slots[:, 0].long()
    assert torch.equal(pages.K.view(-1, d)[at], K_new[:, 0]) and torch.equal(pages.V.view(-1, d)[at], V_new[:, 0])
    # one row: the output is its value, over pages and over the slabs as they are
    Q = torch.randn(1, 2 * H, d, device="cuda").bfloat16()
    cu = dev([0, 1]).int()
    want = V_new[:, 0].repeat_interleave(2, dim=0)[None]
    for over_pages in (True, False):
        out = torch.zeros(1, 2 * H, d, dtype=torch.bfloat16, device="cuda")
        if over_pages:
            gv.gvote_page_attend(p, Q, cu, 1, pages, out, ws)
        else:
            gv.gvote_attend(p, Q, cu, 1, K_new, V_new, cu, (1, 1, 1), out, ws)
        assert torch.equal(out, want)
