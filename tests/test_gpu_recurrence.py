"""The gated linear recurrence and its gradient against float64, within the
bounds that block_reference derives."""
import numpy as np
import pytest
import torch

import paper_2205_11048_amd as gba
from block_reference import BF16, F16, F32, U32, close, matrix, recurrence, recurrence_grad, rounded

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _ws(n, B, D):
    return torch.full((gba.gba_recurrence_workspace_size(n, B, D),), 255, dtype=torch.uint8, device=DEV)


class Case:
    """Inputs, and the two calls."""

    def __init__(self, lengths, D, dtype, pad=0, state=True, tail=0, packed=True, seed=0, gate=1.5):
        rng = np.random.default_rng(len(lengths) * 1009 + D * 31 + seed)
        self.starts = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
        self.used = int(self.starts[-1])
        self.n, self.B, self.D, self.dtype, self.tail = self.used + tail, len(lengths), D, dtype, tail
        self.x, self.x64 = matrix(rng.normal(size=(self.n, D)), dtype, pad)
        self.a, self.a64 = matrix(2.0 + gate * rng.normal(size=(self.n, D)), dtype, 2 * pad)
        self.dh, self.dh64 = matrix(rng.normal(size=(self.n, D)), dtype, pad)
        if tail:   # nothing behind the last sequence is read
            for t in (self.x, self.a, self.dh):
                t[self.used:] = float("nan")
        self.h0 = rng.normal(size=(self.B, D)).astype(np.float32) if state else None
        self.dlast = rng.normal(size=(self.B, D)).astype(np.float32) if state else None
        self.by = dict(offsets=_dev(self.starts)) if packed else dict(length=int(lengths[0]))
        self.pad = pad
        self.ws = _ws(self.n, self.B, D)
        self.err = torch.zeros(1, dtype=torch.int32, device=DEV)

    def new(self):
        wide = torch.full((self.n, self.D + self.pad), 7.0, dtype=self.dtype, device=DEV)
        return wide[:, :self.D]

    def zeros(self):
        return np.zeros((self.B, self.D))

    def forward(self, **kw):
        h = self.new()
        h0 = _dev(self.h0) if self.h0 is not None else None
        last = torch.full((self.B, self.D), float("nan"), device=DEV)
        gba.gba_recurrence(self.x, self.a, h, h0=h0, h_last=last, workspace=self.ws, err=self.err, **self.by, **kw)
        return h, last

    def backward(self, h, **kw):
        dx, da = self.new(), self.new()
        h0 = _dev(self.h0) if self.h0 is not None else None
        dl = _dev(self.dlast) if self.dlast is not None else None
        d0 = torch.full((self.B, self.D), float("nan"), device=DEV)
        gba.gba_recurrence_grad(self.dh, self.x, self.a, h, dx, da, h0=h0, dh_last=dl, dh0=d0, workspace=self.ws,
                                err=self.err, **self.by, **kw)
        return dx, da, d0


def check(c):
    h, last = c.forward()
    h0 = c.h0.astype(np.float64) if c.h0 is not None else c.zeros()
    ref, rlast, E, El = recurrence(c.x64, c.a64, c.starts, h0, c.dtype)
    close(h[:c.used], ref[:c.used], rounded(E, ref, c.dtype)[:c.used], "h")
    close(last, rlast, rounded(El, rlast, F32), "h_last")
    assert (h[c.used:] == 7.0).all()
    dx, da, d0 = c.backward(h)
    h64 = h.double().cpu().numpy()
    dl = c.dlast.astype(np.float64) if c.dlast is not None else c.zeros()
    rx, ra, r0, Ex, Ea, E0 = recurrence_grad(c.dh64, c.x64, c.a64, h64, c.starts, h0, dl, c.dtype)
    close(dx[:c.used], rx[:c.used], rounded(Ex, rx, c.dtype)[:c.used], "dx")
    close(da[:c.used], ra[:c.used], rounded(Ea, ra, c.dtype)[:c.used], "da")
    close(d0, r0, rounded(E0, r0, F32), "dh0")
    for t in (dx, da):
        assert (t[c.used:] == 7.0).all()
    assert int(c.err) == 0
    # the same bits again, without the states' outputs, with the states in place
    again = c.new()
    h0 = _dev(c.h0) if c.h0 is not None else None
    gba.gba_recurrence(c.x, c.a, again, h0=h0, workspace=c.ws, **c.by)
    assert torch.equal(again, h)
    if h0 is not None:
        gba.gba_recurrence(c.x, c.a, again, h0=h0, h_last=h0, workspace=c.ws, **c.by)
        assert torch.equal(again, h) and torch.equal(h0, last)
        carried = _dev(c.dlast)
        dh = c.dh.clone(memory_format=torch.preserve_format) if not c.pad else c.dh
        da2 = c.new()
        gba.gba_recurrence_grad(dh, c.x, c.a, h, dh, da2, h0=_dev(c.h0), dh_last=carried, dh0=carried,
                                workspace=c.ws, **c.by)
        assert torch.equal(carried, d0) and torch.equal(da2, da) and torch.equal(dh[:c.used], dx[:c.used])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("B,L,D,state", [
    (1, 1, 1, True), (3, 1, 5, True), (64, 1, 2048, True), (1, 7, 16, False), (5, 8, 17, True), (2, 129, 64, True),
    (4, 33, 100, False), (3, 65, 256, True), (2, 300, 257, True), (1, 700, 512, True), (300, 3, 8, True),
    (17, 50, 36, True), (9, 64, 1001, False)])
def test_equal_lengths(B, L, D, state, dtype):
    check(Case([L] * B, D, dtype, state=state, packed=False, pad=0 if D % 2 else 3))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [4, 13, 64, 129, 300])
@pytest.mark.parametrize("lengths,tail", [
    ([1], 0), ([0], 3), ([0, 0, 5, 0], 0), ([3, 1, 1, 0, 8, 9, 0], 5), ([64, 0, 63, 65, 1, 127], 1), ([1] * 70, 2),
    ([511, 1, 0, 513], 0)])
def test_packed(lengths, tail, D, dtype):
    check(Case(lengths, D, dtype, tail=tail, pad=1 if D == 13 else 0))


@pytest.mark.parametrize("dtype,D,lengths,tail,packed", [
    # few long sequences, cut into parts
    (F32, 40, [9000], 0, False), (BF16, 64, [12_001], 0, False), (F32, 5, [20_000], 77, True),
    (BF16, 260, [3000, 0, 2999, 1, 1500], 100, True), (F16, 20, [7000] * 3, 0, False), (F32, 64, [0, 9000, 0, 3], 0, True),
    # many ragged ones
    (F32, 16, [(7 * k * k) % 61 for k in range(500)], 11, True),
    (BF16, 72, [(5 * k * k) % 97 for k in range(130)], 0, True)])
def test_long_and_ragged(dtype, D, lengths, tail, packed):
    check(Case(lengths, D, dtype, tail=tail, packed=packed))


@pytest.mark.parametrize("dtype,D", [(F32, 3), (F32, 72), (BF16, 130), (F16, 16)])
def test_one_long_sequence_among_short_ones(dtype, D):
    """A few parts hold many sequences each, the others are passed by one."""
    check(Case([2, 0, 5] * 150 + [6000] + [1, 9, 0, 0] * 100 + [1500], D, dtype, tail=9))


@pytest.mark.parametrize("packed", [False, True])
def test_parts_without_states(packed):
    check(Case([6000, 6000], 24, F32, state=False, packed=packed))


def test_gates_at_their_ends():
    """Gates that hold or forget everything, and long memories: sigmoid(16) leaves 1e-7 a step."""
    n, D = 600, 8
    rng = np.random.default_rng(4)
    c = Case([n], D, F32, packed=False)
    a = np.zeros((n, D))
    a[:, 0], a[:, 1], a[:, 2], a[:, 3] = 200.0, -200.0, float("inf"), -float("inf")
    a[:, 4], a[:, 5], a[:, 6], a[:, 7] = 16.0, -16.0, 80.0 * np.sign(rng.normal(size=n)), 9.0
    c.a, c.a64 = matrix(a, F32)
    check(c)
    h, last = c.forward()
    assert (h[:, [0, 2]] == _dev(c.h0)[:, [0, 2]]).all()                 # kept to the bit
    assert (h[:, [1, 3]] == c.x[:, [1, 3]]).all()                        # forgotten to the bit


def test_a_sequence_keeps_its_infinities():
    lengths = [40, 41, 42]
    for longer in (1, 200):   # whole sequences to a block, and cut into parts
        c = Case([k * longer for k in lengths], 8, F32)
        c.x[c.starts[1] + 3] = float("inf")
        c.x[c.starts[1] + 5] = float("nan")
        h, last = c.forward()
        s = c.starts
        assert torch.isfinite(h[:s[1]]).all() and torch.isfinite(h[s[2]:]).all() and torch.isnan(last[1]).all()
        dx, da, d0 = c.backward(torch.nan_to_num(h, posinf=0.0))
        assert torch.isfinite(dx).all() and torch.isfinite(d0).all()
        c.dh[s[1] + 2] = float("inf")
        dx, da, d0 = c.backward(torch.nan_to_num(h, posinf=0.0))
        assert torch.isfinite(dx[:s[1]]).all() and torch.isfinite(dx[s[2]:]).all()
        assert torch.isfinite(d0[[0, 2]]).all() and not torch.isfinite(d0[1]).any()


def test_the_gradient_is_the_forwards():
    """Along a direction, against central differences of the kernel's own forward in 32 bits: off by what the
    differences leave out, which float64 says, and by the forward's bound over the step."""
    c = Case([30, 1, 50], 12, F32, seed=3)
    rng = np.random.default_rng(8)
    vx, va, v0 = (rng.normal(size=s) for s in (c.x64.shape, c.a64.shape, c.h0.shape))
    h0 = c.h0.astype(np.float64)
    step = 2.0 ** -7
    x64, a64 = c.x64, c.a64
    h, _ = c.forward()
    dx, da, d0 = (t.double().cpu().numpy() for t in c.backward(h))
    along = (dx * vx).sum() + (da * va).sum() + (d0 * v0).sum()
    quotient, plain, noise = 0.0, 0.0, 0.0
    for sign in (1.0, -1.0):
        c.x, xs = matrix(x64 + sign * step * vx, F32)
        c.a, as_ = matrix(a64 + sign * step * va, F32)
        c.h0 = (h0 + sign * step * v0).astype(np.float32)
        h, last = (t.double().cpu().numpy() for t in c.forward())
        quotient += sign * ((h * c.dh64).sum() + (last * c.dlast).sum()) / (2 * step)
        ref, rlast, E, El = recurrence(xs, as_, c.starts, c.h0.astype(np.float64))
        plain += sign * ((ref * c.dh64).sum() + (rlast * c.dlast).sum()) / (2 * step)
        noise += ((rounded(E, ref, F32) * np.abs(c.dh64)).sum() + (rounded(El, rlast, F32) * np.abs(c.dlast)).sum()) / (2 * step)
    rx, ra, r0, Ex, Ea, E0 = recurrence_grad(c.dh64, x64, a64, recurrence(x64, a64, c.starts, h0)[0], c.starts, h0,
                                             c.dlast.astype(np.float64))
    exact = (rx * vx).sum() + (ra * va).sum() + (r0 * v0).sum()
    # (the kernel's gradient takes the rounded h: another u of it in da)
    slack = sum((rounded(e, r, F32) * np.abs(v)).sum() for e, r, v in ((Ex, rx, vx), (Ea, ra, va), (E0, r0, v0)))
    slack += 40 * U32 * (np.abs(ra) * np.abs(va)).sum() + (np.abs(rx) * np.abs(va)).sum() * 40 * U32
    assert abs(along - quotient) <= abs(exact - plain) + noise + slack
    assert abs(exact - plain) < 1e-2 * abs(exact)


def test_step_by_step_is_the_sequence():
    """Serving a sequence one position at a time gives its states, to the bound of the joins."""
    c = Case([24] * 5, 96, F32, packed=False)
    h, last = c.forward()
    state = _dev(c.h0)
    x, a = c.x.reshape(5, 24, 96), c.a.reshape(5, 24, 96)
    ref, _, E, _ = recurrence(c.x64, c.a64, c.starts, c.h0.astype(np.float64))
    bound = rounded(E, ref, F32).reshape(5, 24, 96)
    ws = _ws(5, 5, 96)
    for t in range(24):
        out = torch.empty((5, 96), device=DEV)
        gba.gba_recurrence(x[:, t], a[:, t], out, length=1, h0=state, h_last=state, workspace=ws)
        close(out, ref.reshape(5, 24, 96)[:, t], bound[:, t], f"step {t}")
        assert torch.equal(out, state)


def test_no_positions():
    ws = _ws(0, 3, 6)
    x = torch.empty((0, 6), device=DEV)
    h0, last = torch.randn((3, 6), device=DEV), torch.empty((3, 6), device=DEV)
    off = torch.zeros(4, dtype=torch.int64, device=DEV)
    gba.gba_recurrence(x, x, x, offsets=off, h0=h0, h_last=last, workspace=ws)
    assert torch.equal(last, h0)
    gba.gba_recurrence(x, x, x, offsets=off, h_last=last, workspace=ws)
    assert (last == 0).all()
    d0 = torch.empty_like(h0)
    gba.gba_recurrence_grad(x, x, x, x, x, x, offsets=off, dh_last=h0, dh0=d0, workspace=ws)
    assert torch.equal(d0, h0)
    gba.gba_recurrence(x, x, x, length=4)


@pytest.mark.parametrize("offsets", [[0, 10, 5, 20], [1, 5, 10, 20], [0, 5, 10, 21], [0, 30, 30, 20], [-4, 5, 9, 20],
                                     [0, 5, 10, 1 << 40], [7, 7, 7, 7]])
def test_offsets_out_of_order_are_reported(offsets):
    n, D = 20, 9
    wide = torch.full((n + 8, D), 3.0, device=DEV)
    x, a = torch.randn((n, D), device=DEV), torch.randn((n, D), device=DEV)
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    ws = _ws(n, 3, D)
    for backward in (False, True):
        err = torch.zeros(1, dtype=torch.int32, device=DEV)
        h, out, s = wide[:n], torch.full((n + 8, D), 3.0, device=DEV), torch.zeros((4, D), device=DEV)
        if backward:
            gba.gba_recurrence_grad(x, x, a, a, h, out[:n], offsets=off, dh_last=s[:3], dh0=s[:3], workspace=ws, err=err)
        else:
            gba.gba_recurrence(x, a, h, offsets=off, h0=s[:3], h_last=s[:3], workspace=ws, err=err)
        assert int(err) == gba.DERR_OFFSETS
        assert (wide[n:] == 3.0).all() and (out[n:] == 3.0).all() and (s[3] == 0).all()


@pytest.mark.parametrize("packed", [False, True])
def test_in_a_graph_and_on_another_stream(packed):
    c = Case([900, 900, 900], 40, BF16, packed=packed)
    want = c.forward()
    grads = c.backward(want[0])
    other = torch.cuda.Stream()
    h, last = c.new(), torch.empty((c.B, c.D), device=DEV)
    h0 = _dev(c.h0)
    torch.cuda.synchronize()
    gba.gba_recurrence(c.x, c.a, h, h0=h0, h_last=last, workspace=c.ws, err=c.err, stream=other, **c.by)
    other.synchronize()
    assert torch.equal(h, want[0]) and torch.equal(last, want[1])
    dx, da, d0 = c.new(), c.new(), torch.empty_like(last)
    dl = _dev(c.dlast)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gba.gba_recurrence(c.x, c.a, h, h0=h0, h_last=last, workspace=c.ws, err=c.err, **c.by)
        gba.gba_recurrence_grad(c.dh, c.x, c.a, h, dx, da, h0=h0, dh_last=dl, dh0=d0, workspace=c.ws, err=c.err, **c.by)
    x2 = -c.x
    for k in range(4):
        for t in (h, last, dx, da, d0):
            t.fill_(float("nan"))
        c.x.copy_(-x2 if k % 2 == 0 else x2)
        c.ws.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        if k % 2 == 0:
            for got, ref in zip((h, last, dx, da, d0), (*want, *grads)):
                assert torch.equal(got[:c.used] if got.shape[0] == c.n else got, ref[:c.used] if ref.shape[0] == c.n else ref)
        else:
            eager = c.forward()
            assert torch.equal(h, eager[0]) and torch.equal(last, eager[1])


def test_refusals():
    x = torch.zeros((12, 16), device=DEV)
    s, ws = torch.zeros((3, 16), device=DEV), _ws(12, 3, 16)
    off = torch.tensor([0, 4, 8, 12], device=DEV)
    for bad in [lambda: gba.gba_recurrence(x, x, x.half(), length=4, workspace=ws),
                lambda: gba.gba_recurrence(x, x[:11], x, length=4, workspace=ws),
                lambda: gba.gba_recurrence(x, x, x, length=5, workspace=ws),
                lambda: gba.gba_recurrence(x, x, x, workspace=ws),
                lambda: gba.gba_recurrence(x, x, x, length=4),
                lambda: gba.gba_recurrence(x, x, x, offsets=off, length=4, workspace=ws),
                lambda: gba.gba_recurrence(x, x, x, offsets=off[:1], workspace=ws),
                lambda: gba.gba_recurrence(x, x, x, offsets=off.int(), workspace=ws),
                lambda: gba.gba_recurrence(x, x, x, length=4, h0=s[:2], workspace=ws),
                lambda: gba.gba_recurrence(x, x, x, length=4, h_last=s.half(), workspace=ws),
                lambda: gba.gba_recurrence(x, x, x, length=4, workspace=ws[:-1]),
                lambda: gba.gba_recurrence(x.T, x.T, x.T, length=4, workspace=ws),
                lambda: gba.gba_recurrence_grad(x, x, x, x, x, x.cpu(), length=4, workspace=ws),
                lambda: gba.gba_recurrence_grad(x, x, x, x.half(), x, x, length=4, workspace=ws),
                lambda: gba.gba_recurrence_grad(x, x, x, x, x, x, length=4, dh0=s[:, :15], workspace=ws),
                lambda: gba.gba_recurrence_workspace_size(12, 0, 16), lambda: gba.gba_recurrence_workspace_size(-1, 1, 16)]:
        with pytest.raises(gba.GBAError):
            bad()


def test_rows_far_apart_and_many():
    """Strides of 2^22 elements (more than 2^32 bytes from the first row to the last), and more than 2^31 elements."""
    c = Case([150] * 4, 40, BF16, packed=False)
    want, last = c.forward()
    dx, da, d0 = c.backward(want)
    far = torch.empty(600 << 22, dtype=BF16, device=DEV).as_strided((600, 40), (1 << 22, 1))
    far.copy_(c.x)
    near, c.x = c.x, far
    h, _ = c.forward()
    assert torch.equal(h, want)
    assert torch.equal(c.backward(want)[1], da)
    c.x = near
    gba.gba_recurrence(c.x, c.a, far, h0=_dev(c.h0), workspace=c.ws, **c.by)
    assert torch.equal(far, want)
    del far
    n, D, L = 3 << 23, 90, 64
    x, a = (torch.randn((L, D), device=DEV).to(BF16) for _ in range(2))
    h = torch.empty_like(x)
    gba.gba_recurrence(x, a, h, length=L, workspace=_ws(L, 1, D))
    bound = 2 * 36 * 64 * U32   # (tiles lie elsewhere in the sequences: each is within 36 u a step of the exact state)
    X, A = (t.repeat(n // L, 1) for t in (x, a))
    ws = _ws(n, n // L, D)
    for packed in (False, True):
        by = dict(offsets=torch.arange(0, n + 1, L, device=DEV)) if packed else dict(length=L)
        H = torch.full_like(X, float("nan"))
        gba.gba_recurrence(X, A, H, workspace=ws, **by)
        # (in bf16 the states are an ulp apart where they lie next to a border)
        for part in H.view(n // L, L, D).split(1 << 16):
            assert ((part.float() - h.float()).abs() <= 2.0 ** -7 * h.float().abs() + 8 * bound).all()
