"""The head's arrays anywhere that they may lie: x, w, dx and dw 16 bytes into an allocation, the others 4; the results are
the same, bit for bit, and what lies around them stays as it was.
"""
import pytest
import torch

import paper_2411_12364_amd as U

from .test_gpu_head import BF, F, desc, make, scratch

pytestmark = pytest.mark.gpu


def placed(t, lead, room):
    """A copy of the tensor `lead` bytes past a multiple of 256, with 64 bytes of 0x5A before and after it."""
    n = t.numel() * t.element_size()
    raw = torch.full((n + 1024,), 0x5A, dtype=torch.uint8, device="cuda")
    first = -raw.data_ptr() % 256 + 256 + lead
    here = raw[first:first + n]
    here.copy_(t.contiguous().reshape(-1).view(torch.uint8))
    room.append((raw, first, n))
    return here.view(t.dtype).view(t.shape)


@pytest.mark.parametrize("xt,gt", [(F, F), (F, BF), (BF, F), (BF, BF)])
@pytest.mark.parametrize("T,vocab,d", [(1, 3, 8), (5, 70, 24), (70, 300, 72), (300, 513, 136), (1030, 700, 264)])
def test_places(T, vocab, d, xt, gt):
    print(f"[case] head {T} {vocab} {d} {xt} {gt}", flush=True)
    x, w, y, dloss = make(T, vocab, d, xt, none=0.3)
    ds = desc(vocab, d, xt, gt, 0.7)
    got = []
    for big, small in ((0, 0), (16, 4), (48, 12), (112, 8)):
        room = []
        at = lambda t, lead: placed(t, lead, room)                      # noqa: E731
        X, W, Y, G = at(x, big), at(w, big), at(y, small), at(dloss, small)
        loss, lse = at(torch.full((T,), 9.0, device="cuda"), small), at(torch.full((T,), 9.0, device="cuda"), small)
        dx = at(torch.full_like(x, 9.0), big)
        dw = at(torch.full(w.shape, 0.25, dtype=gt, device="cuda"), big)
        ws = scratch(U.umem_head_loss_workspace_size, ds, T)
        U.check(U.umem_head_loss(ds, T, X, W, Y, loss, lse, ws, ws.numel()))
        ws = scratch(U.umem_head_backward_workspace_size, ds, T)
        U.check(U.umem_head_backward(ds, T, X, W, Y, lse, G, dx, dw, int(gt == F), ws, ws.numel()))
        for raw, first, n in room:
            assert bool((raw[first - 64:first] == 0x5A).all()) and bool((raw[first + n:first + n + 64] == 0x5A).all())
        for a, b in ((X, x), (W, w), (Y, y), (G, dloss)):
            assert torch.equal(a, b)
        got.append([t.clone() for t in (loss, lse, dx, dw)])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
