"""Plain float64 forms of the recurrence, the norms with gate and residual, and
the AdamW step, with the bounds of what 32 bits may leave: shared by the tests
of those operators."""
import numpy as np
import torch

U32 = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -148, BF16: 2.0 ** -133, F16: 2.0 ** -24}


def rounded(bound, ref, dtype):
    """The bound of a value that is rounded to ``dtype`` at the end."""
    return 1.01 * bound + 1.01 * ROUND[dtype] * (np.abs(ref) + bound) + TINY[dtype]


def close(got, ref, bound, name):
    got = got.detach().double().cpu().numpy()
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (name, int(bad.sum()), got[bad][:3], ref[bad][:3], np.broadcast_to(bound, ref.shape)[bad][:3])


def matrix(x64, dtype, pad=0, device="cuda"):
    """A matrix inside a wider one that holds NaN beside it, and its values."""
    n, D = x64.shape
    x = torch.from_numpy(x64).to(dtype)
    wide = torch.full((n, D + pad), float("nan"), dtype=dtype)
    wide[:, :D] = x
    return wide.to(device)[:, :D], x.double().numpy()


# ------------------------------------------------------------- the recurrence
def sigmoids(a):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-a)), 1.0 / (1.0 + np.exp(a))


# A step's gate is off by at most 8 u of the smaller of f and 1 - f (the power of two 3 u, the sum, the reciprocal 2 u
# and the product); a step adds the difference's rounding and its own.  Where maps of steps are joined F is a product of
# f's, off by 9 u a step, and each join (fewer than 20 a tile) rounds once.  With A the recurrence of magnitudes, 12 u A a
# step and 24 u A for the joins bound it.  With 16-bit inputs the power of two is taken of a * log2(e) as it is rounded: the
# smaller of f and 1 - f is off by |a| u more, f (of which it is the whole, or the part 1 - f) by as much of itself at most.
STEP = 36 * U32


def gate_error(a, dtype):
    return np.zeros_like(a) if dtype == F32 else np.abs(a) * U32


def recurrence(x, a, starts, h0, dtype=F32):
    """h, the last states and their bounds; sequence b holds positions starts[b] .. starts[b + 1] - 1."""
    f, i = sigmoids(a)
    more = gate_error(a, dtype)
    h, E = np.zeros_like(x), np.zeros_like(x)
    last, E_last = h0.copy(), np.zeros_like(h0)
    for b in range(len(starts) - 1):
        s, A, e = h0[b], np.abs(h0[b]), 0.0
        for t in range(starts[b], starts[b + 1]):
            s = f[t] * s + i[t] * x[t]
            A = f[t] * A + i[t] * np.abs(x[t])
            e = f[t] * e + (STEP + more[t]) * A
            h[t], E[t] = s, e
        if starts[b + 1] > starts[b]:
            last[b], E_last[b] = s, e
    return h, last, E, E_last


def recurrence_grad(dh, x, a, h, starts, h0, dlast, dtype=F32):
    """dx, da, dh0 and their bounds."""
    f, i = sigmoids(a)
    more = gate_error(a, dtype)
    dx, da, Ex, Ea = (np.zeros_like(x) for _ in range(4))
    d0, E0 = dlast.copy(), np.zeros_like(dlast)
    for b in range(len(starts) - 1):
        c, C, e = dlast[b], np.abs(dlast[b]), 0.0
        for t in range(starts[b + 1] - 1, starts[b] - 1, -1):
            g, G = dh[t] + c, np.abs(dh[t]) + C
            eg = e + 2 * U32 * G
            before = h[t - 1] if t > starts[b] else h0[b]
            dx[t], Ex[t] = i[t] * g, i[t] * eg + (10 * U32 + more[t]) * i[t] * G
            diff, D = before - x[t], np.abs(before) + np.abs(x[t])
            da[t] = g * diff * f[t] * i[t]
            Ea[t] = (np.abs(diff) * eg + (22 * U32 + 2 * more[t]) * G * D) * f[t] * i[t]
            c, C = f[t] * g, f[t] * G
            e = f[t] * eg + (STEP + more[t]) * C
        if starts[b + 1] > starts[b]:
            d0[b], E0[b] = c, e
    return dx, da, d0, Ex, Ea, E0


# ------------------------------------------- norms with gate and residual
def row_statistics(x, kind, eps):
    mean = x.mean(1, keepdims=True) if kind == "layer" else np.zeros((x.shape[0], 1))
    return mean, 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)


def normed(x, kind, w, b, eps):
    if kind == "none":
        return x
    mean, rstd = row_statistics(x, kind, eps)
    return (x - mean) * rstd * w + b


def gate_factor(gate, kind, rows):
    """The factor of each row and its derivative by the gate."""
    if kind == "none":
        return np.ones((1, 1)), np.zeros((1, 1))
    g = gate[rows]
    if kind == "linear":
        return g, np.ones_like(g)
    s, c = sigmoids(g)
    return s, s * c


def norm_grad(d, v, kind, w, mean, rstd):
    """What reaches v from d, the gradient of its norm (v normalised as well)."""
    if kind == "none":
        return d, v
    vh = (v - mean) * rstd
    k = d * w
    m = k.mean(1, keepdims=True) if kind == "layer" else 0.0
    return rstd * (k - m - vh * (k * vh).mean(1, keepdims=True)), vh


# ------------------------------------------------------------------- AdamW
def mix_bits(x):
    x = x.astype(np.uint64)
    low = np.uint64(0xFFFFFFFF)
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(0xB7E15163)) & low
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(0x9E3779B1)) & low
    return x ^ (x >> np.uint64(16))


def random_words(n, seed, t, tensor):
    """16 bits for m and 16 for v's root, for each element of a tensor."""
    low = np.uint64(0xFFFFFFFF)
    one = np.array([(seed + t) & 0xFFFFFFFF], dtype=np.uint64)
    key = mix_bits((mix_bits(one) + np.uint64(tensor)) & low)
    j = np.arange(n, dtype=np.uint64)
    bits = mix_bits((mix_bits((key + (j >> np.uint64(8))) & low) + (j & np.uint64(255))) & low)
    return bits & np.uint64(0xFFFF), bits >> np.uint64(16)


def decode(code, exp, mantissa):
    """What codes stand for, by the formula of the header."""
    code = code.astype(np.int64)
    sign = np.where(code >> 7, -1.0, 1.0) if mantissa == 3 else 1.0
    code = code & (127 if mantissa == 3 else 255)
    k, i = code >> mantissa, code & ((1 << mantissa) - 1)
    E = np.repeat(exp.astype(np.int64), 256)[:len(code)]
    return sign * np.exp2(E - 127.0) * np.exp2(np.maximum(k, 1) - 15.0) * ((k > 0) + i / 2.0 ** mantissa)


def encode(x, mantissa, words):
    """Codes and exponents of float32 values."""
    n = len(x)
    top = np.zeros(-(-n // 256) * 256)
    top[:n] = np.abs(x.astype(np.float64))
    top = top.reshape(-1, 256).max(1)
    most = 2.0 - 2.0 ** -mantissa
    exp = np.full(len(top), -126)
    for e in range(-126, 128):
        exp = np.where(top > most * 2.0 ** (e - 1), e, exp)
    exp = np.where(top > 0, np.maximum(exp, -126) + 127, 0)
    y = np.abs(x.astype(np.float64)) * np.exp2(127.0 - np.repeat(exp, 256)[:n])
    with np.errstate(divide="ignore"):
        e = np.where(y > 0, np.maximum(np.floor(np.log2(np.where(y > 0, y, 1.0))), -14), -14)
    places = 23 - mantissa
    f = np.rint(y * np.exp2(mantissa + places - e)) * 2.0 ** -places   # (even on a tie)
    f = np.floor(f + (words.astype(np.float64) + 0.5) * 2.0 ** -16)
    code = np.minimum(f + (e + 14) * 2 ** mantissa, 2 ** (4 + mantissa) - 1).astype(np.int64)
    if mantissa == 3:
        code += 128 * (x < 0)
    return code.astype(np.uint8), exp.astype(np.uint8)
