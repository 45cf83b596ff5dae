"""A step number on the device that is below 1 counts as 1: in the constants and in
the rounding of moments in 8 bits."""
import pytest
import torch

import paper_2205_11048_amd as gba
from block_reference import BF16, F16, F32
from test_gpu_adamw import DEV, HP, Case

pytestmark = pytest.mark.gpu


def _step(eight, t, t_device):
    c = Case([3000, 41], [BF16, F32], eight, copies=[F16, None])
    on_device = None if t_device is None else torch.tensor([t_device], device=DEV)
    gba.gba_adamw(c.list, **HP, t=t, t_device=on_device, seed=3, err=c.err)
    assert int(c.err) == 0
    return [*c.p, *c.m, *c.v, c.copies[0]] + ([*c.me, *c.ve] if eight else [])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("below", [0, -5, -(1 << 62)])
def test_a_number_below_one_is_the_first_step(below, eight):
    first = _step(eight, 1, None)
    assert all(torch.equal(a, b) for a, b in zip(_step(eight, 99, below), first))
    assert all(torch.equal(a, b) for a, b in zip(_step(eight, 99, 1), first))
    assert not torch.equal(_step(eight, 99, 2)[0], first[0])
