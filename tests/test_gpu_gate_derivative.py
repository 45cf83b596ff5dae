"""The gradient of sigmoid gates that are nearly open or nearly closed, with a bound
relative to the derivative alone: s (1 - s) falls to 1e-13 at gates of 30, on both sides.

Without norms dgate = d * sum of dh * z over the rows that share the gate, d = l (1 - l) with l the smaller of s and
1 - s: 1 / (1 + t) or t / (1 + t), t = exp(-g).  In 32 bits (unit roundoff u): t is off by 2 u, of which l takes the
part 1 - l; the sum, the quotient and the product with t round l by u each; d takes the part (1 - 2 l) / (1 - l) of
l's error, no more than all of it, and rounds twice: 7 u.  (As s (1 - s), with both from t: 8 u.)  Below the normal
numbers l and d are off by half of the least number more, 2^-150 each.  The sum's terms, and the sum with d, round
3 + count times."""
import numpy as np
import pytest
import torch

from block_reference import BF16, F16, F32, ROUND, TINY, U32, close, matrix, sigmoids
from test_gpu_residual_norm import Case

GATES = np.array([-88.0, -30.0, -17.0, -16.0, -12.0, -8.0, -1.0, 0.0, 0.5, 4.0, 8.0, 12.0, 16.0, 17.0, 20.0, 30.0, 60.0, 80.0])


@pytest.mark.gpu
@pytest.mark.parametrize("gtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,D,span", [
    (40, 3, 1), (300, 136, 1), (9, 3000, 1), (5, 5000, 1),           # a gate for each row
    (40, 3, 7), (300, 136, 100), (70, 2100, 35), (12, 6000, 6),      # units of the rows that share one
    (1100, 600, 2), (4801, 24, 3),                                   # units in turn, a gate for each group of lanes
    (5, 9000, 1), (7, 9000, 4)])                                     # rows read again
def test_gates_at_their_ends(n, D, span, gtype):
    c = Case(n, D, F32, F32, gate="sigmoid", span=span, gtype=gtype, post="none", pre="none", weights=False, bias=False)
    rng = np.random.default_rng(n + D)
    c.g, c.g64 = matrix(rng.choice(GATES, c.g64.shape), gtype)
    assert np.isin(c.g64, GATES).all()
    dg = torch.full_like(c.g, float("nan"))
    c.backward(None, {}, dgate=dg)
    s, rest = sigmoids(c.g64)
    terms = c.dh64 * c.z64
    total, size, count = (np.zeros(c.g64.shape) for _ in range(3))
    for to, val in ((total, terms), (size, np.abs(terms)), (count, np.ones_like(terms))):
        np.add.at(to, c.rows, val)
    d = s * rest
    ref = total * d
    bound = 1.01 * U32 * (8 * np.abs(ref) + (count + 3) * size * d) + 2.0 ** -149 * size
    # (TINY: what a type holds below its normal numbers is off by half of its least one; 16 bits get there soon)
    close(dg, ref, 1.01 * bound + 1.01 * ROUND[gtype] * (np.abs(ref) + bound) + TINY[gtype], "dgate")


def test_the_derivative_against_differences():
    """Of the sigmoid of -g, which keeps its digits where that of g is next to 1; a step of 1e-4 leaves out 1e-8 / 6
    of the third derivative, which is no more than the first one."""
    g, e = GATES[GATES >= 0.0], 1e-4
    quotient = (sigmoids(g - e)[1] - sigmoids(g + e)[1]) / (2 * e)
    s, rest = sigmoids(g)
    assert (np.abs(quotient - s * rest) <= 1e-8 * s * rest).all()
    assert np.allclose(np.multiply(*sigmoids(-g)), s * rest, rtol=1e-14, atol=0.0)
