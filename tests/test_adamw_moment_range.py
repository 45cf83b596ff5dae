"""How far apart the elements of one block of 8-bit moments may be: what the header says of it, on the float64 form of
the codes and on the kernel.

The least code of m, d, is 2^-17, that of v's root, c, 2^-18 of 2^(E - 127).  A root below c may become 0 and leave an
m behind.  Then every gradient since has been below c / sqrt(1 - b2) = 32 c (a larger one would have brought a root of
c or more, which is never rounded to 0), and m is below that and what its own roundings left: each has a deviation of
no more than half the distance of two codes, here d, and m remembers 1 / (1 - b1^2) = 5.3 of them, so 2.3 d, six times
of which is 14 d.  With eps no less than c and d (here c < d) the step is no more than (32 c + 14 d) / eps < 46 lr,
whatever the elements are, beside the new gradient's own (1 - b1) / sqrt(1 - b2) = 3.2 lr; with eps far below it is
thousands of lr.  At gradients of 2^-12 of
the block's largest a root has 16 codes to an octave; it goes down by 1 / 2000 of itself a step, by chance in steps of
1 / 16, whose variance over the 1000 steps that it remembers is 1000 / 2000 / 16 of its square, 18 % of itself: the
largest of some thousand steps is less than twice that of moments in 32 bits."""
import numpy as np
import pytest
import torch

import paper_2205_11048_amd as gba
from block_reference import decode, encode, random_words

B1, B2, SIGMA, STEPS, BLOCKS = 0.9, 0.999, 1e-2, 600, 8
N = 256 * BLOCKS
SMALL = np.arange(N) % 256 >= 128


def gradients(ratio):
    rng = np.random.default_rng(7)
    scale = np.where(SMALL, ratio, 1.0) * SIGMA
    for _ in range(STEPS):
        yield (scale * rng.normal(size=N)).astype(np.float32)


def largest_exact(ratio, eps):
    """The largest step of the small elements with moments in 64 bits, over lr."""
    m, v, worst = np.zeros(N), np.zeros(N), 0.0
    for t, g in enumerate(gradients(ratio), 1):
        g = g.astype(np.float64)
        m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
        worst = max(worst, np.abs(m / (1 - B1 ** t) / (np.sqrt(v / (1 - B2 ** t)) + eps))[SMALL].max())
    return worst


def steps_of_codes(ratio, eps):
    f = np.float32
    m, v, me, ve = (np.zeros(k, np.uint8) for k in (N, N, BLOCKS, BLOCKS))
    for t, g in enumerate(gradients(ratio), 1):
        mn = f(B1) * decode(m, me, 3).astype(f) + f(1 - B1) * g
        vn = f(B2) * np.square(decode(v, ve, 4).astype(f)) + f(1 - B2) * (g * g)
        yield mn / (1 - B1 ** t) / (np.sqrt(vn) / np.sqrt(1 - B2 ** t) + eps)
        wm, wv = random_words(N, 1, t, 0)
        (m, me), (v, ve) = encode(mn, 3, wm), encode(np.sqrt(vn), 4, wv)


def steps_of_kernel(ratio, eps):
    p, g = (torch.zeros(N, device="cuda") for _ in range(2))
    m, v, me, ve = (torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (N, N, BLOCKS, BLOCKS))
    tensors = gba.gba_adamw_list([p], [g], [m], [v], [me], [ve])
    for t, step in enumerate(gradients(ratio), 1):
        g.copy_(torch.from_numpy(step))
        p.zero_()
        gba.gba_adamw(tensors, 1.0, B1, B2, eps, 0.0, t, seed=1)
        yield p.cpu().numpy()


def check(steps):
    for ratio in (1.0, 2.0 ** -8, 2.0 ** -12):
        for eps in (1e-8, 1e-12):
            worst = max(np.abs(s[SMALL]).max() for s in steps(ratio, eps))
            assert worst < 2 * largest_exact(ratio, eps), (ratio, eps, worst)
    # (the block's largest m and root stay below 2^-6 here, and the least codes no more than 2^-23 and 2^-24)
    for ratio in (2.0 ** -14, 2.0 ** -16, 2.0 ** -18, 2.0 ** -22, 2.0 ** -30):
        worst = max(np.abs(s[SMALL]).max() for s in steps(ratio, 2.0 ** -23))
        assert worst < 46 + 3.2, (ratio, worst)


def test_steps_of_the_codes():
    check(steps_of_codes)


@pytest.mark.gpu
def test_steps_of_the_kernel():
    check(steps_of_kernel)


@pytest.mark.parametrize("mantissa", [3, 4])
def test_what_the_least_code_holds(mantissa):
    """From the least code's value on nothing is rounded to 0; below it by chance."""
    least = 2.0 ** -(14 + mantissa)
    for word in (0, 40_000, 65_535):
        value = np.array([1.0, least, 1.5 * least, 0.5 * least], np.float32)
        code, exp = encode(value, mantissa, np.full(4, word))
        assert exp[0] == 127 and (code[1:3] > 0).all() and (code[3] > 0) == (word >= 32_768)
