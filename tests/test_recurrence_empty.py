"""Sequences of no positions at all through the C entry, with offsets NULL: an empty
sequence's last state is its first one, and its state's gradient passes as it is."""
import pytest
import torch

import paper_2205_11048_amd as gba
from test_block_host import _scan, _scan_grad
from test_worker_host import HIP, OK, P, fake, no_gpu


@no_gpu
def test_host_paths():
    """A launch where there is something to write, and none otherwise."""
    L = gba.lib()
    none = dict(n=0, x=None, a=None, h=None)
    assert _scan(L, **none) == OK
    assert _scan(L, h0=fake(8), **none) == OK
    assert _scan(L, last=fake(9), **none) == HIP
    assert _scan(L, h0=fake(8), last=fake(9), **none) == HIP
    assert _scan(L, h0=fake(8), last=fake(8), **none) == OK
    none.update(dh=None, dx=None, da=None)
    assert _scan_grad(L, **none) == OK
    assert _scan_grad(L, h0=fake(7), dl=fake(8), **none) == OK
    assert _scan_grad(L, d0=fake(9), **none) == HIP
    assert _scan_grad(L, dl=fake(8), d0=fake(9), **none) == HIP
    assert _scan_grad(L, dl=fake(8), d0=fake(8), **none) == OK


@pytest.mark.gpu
@pytest.mark.parametrize("B,D", [(1, 1), (3, 7), (5, 130), (4097, 64), (70_001, 33)])
def test_states(B, D):
    L, stream = gba.lib(), torch.cuda.current_stream().cuda_stream
    ws = torch.empty(gba.gba_recurrence_workspace_size(0, B, D), dtype=torch.uint8, device="cuda")
    wide = torch.empty(B * D + 2, device="cuda")
    out, state = wide[1:-1], torch.randn(B * D, device="cuda")   # (out at an element's alignment)

    def forward(h0, last):
        return L.gba_recurrence(None, D, None, D, 0, 0, B, D, None, h0, None, D, last, P(ws.data_ptr()), ws.numel(), None, stream)

    def backward(dl, d0):
        return L.gba_recurrence_grad(None, D, None, D, None, D, None, D, 0, 0, B, D, None, None, dl, None, D, None, D, d0,
                                     P(ws.data_ptr()), ws.numel(), None, stream)

    for call in (forward, backward):
        for given in (True, False):
            wide.fill_(5.0)
            assert call(P(state.data_ptr()) if given else None, P(out.data_ptr())) == OK
            assert torch.equal(out, state) if given else (out == 0).all()
            assert float(wide[0]) == 5.0 and float(wide[-1]) == 5.0
        before = state.clone()
        assert call(P(state.data_ptr()), P(state.data_ptr())) == OK
        assert torch.equal(state, before)
