"""A gate's span below 1 is refused by both directions, with a gate and without."""
import pytest
import torch

import paper_2205_11048_amd as gba

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("span", [0, -1, -7])
@pytest.mark.parametrize("gated", [False, True])
def test_spans_below_one(span, gated):
    x, s = torch.zeros((6, 16), device="cuda"), torch.zeros(6, device="cuda")
    g = torch.ones((6, 16), device="cuda") if gated else None
    ws = torch.empty(gba.gba_residual_norm_grad_workspace_size(6, 16), dtype=torch.uint8, device="cuda")
    for call in (lambda **kw: gba.gba_residual_norm(x, x, x, x, **kw),
                 lambda **kw: gba.gba_residual_norm_grad(x, x, x, x, x, x, ws, post_rstd=s, pre_rstd=s, **kw),
                 lambda **kw: gba.gba_residual_norm_grad(x, x, x, x, x, x, ws, post_rstd=s, pre_rstd=s, dgate=g, **kw)):
        with pytest.raises(gba.GBAError):
            call(gate=g, gate_span=span)
