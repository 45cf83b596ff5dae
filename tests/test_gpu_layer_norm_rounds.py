"""Layer norm and its gradient where blocks take rows in more than one round,
and at every shape of a row over the threads, against float64: the bounds are
those of the other sizes."""
import pytest
import torch

import test_gpu_layer_norm as base

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16

# n, D, type, weight type, parameters, pad, shift of the values
FORWARD_ROUNDS = [   # more than 2048 blocks' rows
    (1_100_003, 3, F32, F32, "wb", 0, 0.0),     # narrower than a vector
    (600_011, 20, BF16, F32, "wb", 0, 0.0),
    (16_500, 520, BF16, BF16, "wb", 1, 0.0),
    (9001, 1300, F32, F32, "wb", 0, 0.5),       # two waves a row
    (2100, 8000, F32, F32, "w", 0, 0.0),        # a block a row
]
BACKWARD_ROUNDS = [   # more than 512 blocks' rows
    (100_003, 40, F32, F32, "wb", 0, 0.0),
    (270_001, 7, BF16, F32, "wb", 0, 0.0),      # narrower than a vector
    (9000, 520, BF16, BF16, "w", 1, 0.0),
    (2500, 2048, F32, F32, "wb", 0, 0.5),       # four waves a row
    (1100, 8192, BF16, F32, "wb", 0, 0.0),      # a block a row
    (1101, 7003, F32, F32, "wb", 3, 0.0),
]
WIDE = [   # rows read again, and more of them than one partial sum takes
    (300, 8200, BF16, F32, "wb", 0, 0.0), (700, 10_007, F32, F32, "wb", 0, 0.0), (513, 9000, F16, F16, "w", 2, 0.0),
    (260, 17_001, BF16, BF16, "wb", 0, 0.0)]
WIDTHS = [300, 600, 1001, 1300, 2048, 3000, 4096, 6000, 8000, 12_000, 16_381]


@pytest.mark.parametrize("n,D,dtype,wtype,which,pad,shift", FORWARD_ROUNDS + WIDE)
def test_forward_rounds(n, D, dtype, wtype, which, pad, shift):
    base.test_forward(n, D, dtype, wtype, which, pad, shift)


@pytest.mark.parametrize("n,D,dtype,wtype,which,pad,shift", BACKWARD_ROUNDS + WIDE)
def test_backward_rounds(n, D, dtype, wtype, which, pad, shift):
    base.test_backward(n, D, dtype, wtype, which, pad, shift)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("D", WIDTHS)
def test_widths(D, dtype):
    base.test_forward(37, D, dtype, F32, "wb", 0, 0.0)
    base.test_backward(37, D, dtype, F32, "wb", 0, 0.0)
