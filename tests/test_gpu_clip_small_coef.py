"""Clipping where the coefficient is below float32's normal range, against float64.

Tolerances.  An element takes the coefficient's rounding to 24 bits, the
product's and the store's in its type (u = 2^-24, u_t): (2 u + u_t) of its
magnitude, widened by a percent; a result below the type's normal range half its
smallest subnormal, twice."""
import math

import numpy as np
import pytest
import torch

import paper_2205_11048_amd as gba

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}


@pytest.mark.parametrize("scale,max_norm,types,outs_types", [
    (1e38, 1.0, [F32], [F32]),
    (1e38, 1.0, [BF16, F32], [F32, F16]),
    (1e37, 1e-3, [F32, BF16], [BF16, F32]),
    (3e30, 1e-12, [F32], [F32]),
    (1.0, 1e-38, [F32], [F32]),
    (1e-3, 1e-42, [F32], [F32]),
    (1e38, 0.1, [F32], [F32]),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_small_coefficients(scale, max_norm, types, outs_types, in_place):
    rng = np.random.default_rng(7)
    # (uniform: no element passes the type's range)
    grads = [torch.from_numpy((rng.uniform(-1, 1, s) * scale).astype(np.float32)).to(types[i % len(types)]).to(DEV)
             for i, s in enumerate((70_001, 8192, 13, 40_000))]
    g64 = [g.double().cpu().numpy() for g in grads]
    outs = grads if in_place else [torch.full(g.shape, 7.0, dtype=outs_types[i % len(outs_types)], device=DEV)
                                   for i, g in enumerate(grads)]
    tensors = gba.gba_tensor_list(grads, outs)
    norm, coef = torch.full((1,), -1.0, device=DEV), torch.full((1,), -1.0, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.full((gba.gba_grad_norm_workspace_size(tensors),), 255, dtype=torch.uint8, device=DEV)
    gba.gba_clip_grads(tensors, max_norm, norm, ws, coef=coef, err=err)
    exact = math.sqrt(sum(float((g * g).sum()) for g in g64))
    c = max_norm / exact
    assert c < 2.0 ** -126 and int(err) == 0
    assert abs(float(coef) - c) <= 2.0 ** -149   # reported in float32
    for g, o in zip(g64, outs):
        ref, got = g * c, o.double().cpu().numpy()
        bound = 1.01 * (2 * 2.0 ** -24 + ROUND[o.dtype]) * np.abs(ref) + TINY[o.dtype]
        assert (np.abs(got - ref) <= bound).all(), float((np.abs(got - ref) / np.abs(ref)).max())
