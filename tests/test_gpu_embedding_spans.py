"""The embedding gradient of many tokens of narrow rows, whose lane groups take
8 to 32 positions each, several batches of rows after one another: against
float64, with the bounds of the other sizes."""
import pytest
import torch

import test_gpu_embedding as base

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("n,R,D,dtype,out_type,pattern,padding,pad", [
    (300_007, 50_000, 16, BF16, F32, "zipf", 3, 0),          # two lanes a row, 8 positions
    (300_001, 200_000, 32, BF16, F32, "zipf", 0, 1),         # four, 16
    (290_003, 3, 32, BF16, F32, "same", -1, 0),
    (270_001, 400_000, 29, F16, BF16, "zipf", 12, 0),
    (150_001, 40_000, 64, BF16, BF16, "zipf", 39_999, 0),    # eight, 16
    (300_000, 7, 64, BF16, F32, "zipf", 2, 0),               # ... 32
    (150_003, 20_000, 64, F32, F32, "zipf", -1, 0),          # sixteen, 32
    (140_009, 150_000, 50, F32, F32, "distinct", 5, 3),
    (100_001, 9000, 128, F32, F32, "zipf", 1, 0),            # thirty-two, 32
    (70_001, 5000, 300, BF16, F32, "zipf", 4, 0),            # a wave, 32
])
def test_gradient_of_many_tokens(n, R, D, dtype, out_type, pattern, padding, pad):
    base.test_gradient(n, R, D, dtype, out_type, pattern, padding, pad)
