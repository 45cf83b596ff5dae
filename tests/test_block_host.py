"""Host paths of the recurrence, the norms with gate and residual, and the AdamW
step on a machine without a GPU: argument checks, size queries, the list, each
call with fake device addresses up to its first launch, which fails because there
is no device; and the float64 forms that the GPU tests compare with, against
differences."""
import ctypes

import numpy as np
import pytest

import block_reference as ref
import paper_2205_11048_amd as gba
from test_worker_host import BF16, F16, F32, HIP, INVALID, NULL, OK, P, SIZE, WORKSPACE, fake, no_gpu


def _scan(L, n=12, B=3, D=16, t=BF16, xs=16, as_=16, hs=16, x=fake(0), a=fake(1), h=fake(2), off=None, h0=None, last=None,
          work=fake(3), ws=None):
    ws = 1 << 50 if ws is None else ws
    return L.gba_recurrence(x, xs, a, as_, t, n, B, D, off, h0, h, hs, last, work, SIZE(ws), None, None)


def _scan_grad(L, n=12, B=3, D=16, t=BF16, s=16, dxs=16, dh=fake(0), x=fake(1), a=fake(2), h=fake(3), dx=fake(4), da=fake(5),
               off=None, h0=None, dl=None, d0=None, work=fake(6), ws=None):
    ws = 1 << 50 if ws is None else ws
    return L.gba_recurrence_grad(dh, s, x, s, a, s, h, s, t, n, B, D, off, h0, dl, dx, dxs, da, s, d0, work, SIZE(ws), None, None)


SIZES = [(1, 1, 1), (64, 64, 2048), (32_768, 32, 2048), (100_000, 1, 511), (205_000, 4_100, 64), ((1 << 31) - 1, 1, 1 << 20)]


@no_gpu
@pytest.mark.parametrize("n,B,D", SIZES)
@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_recurrence_host_paths(n, B, D, t):
    L = gba.lib()
    need = gba.gba_recurrence_workspace_size(n, B, D)
    s = dict(n=n, B=B, D=D, t=t)
    for off in (None, fake(7)):
        if off is None and n % B:
            continue
        assert _scan(L, xs=D, as_=D, hs=D, off=off, h0=fake(8), last=fake(8), ws=need, **s) == HIP
        assert _scan(L, xs=D, as_=D, hs=D, off=off, ws=need - 1, **s) == WORKSPACE
        assert _scan_grad(L, s=D, dxs=D, off=off, dl=fake(8), d0=fake(8), ws=need, **{k: v for k, v in s.items()}) == HIP
        assert _scan_grad(L, s=D, dxs=D, off=off, ws=need - 1, **s) == WORKSPACE
    assert _scan(L, n=0, B=B, D=D, xs=D, as_=D, hs=D, x=None, a=None, h=None) == OK


def test_recurrence_refusals():
    L = gba.lib()
    for kw in (dict(n=-1), dict(n=1 << 31), dict(B=0), dict(B=1 << 31), dict(B=5), dict(D=0), dict(D=(1 << 20) + 1, xs=1 << 21),
               dict(t=3), dict(xs=15), dict(as_=15), dict(hs=15), dict(x=fake(0, 1)), dict(h=fake(2, 1)), dict(h0=fake(4, 2)),
               dict(last=fake(4, 2)), dict(off=fake(4, 4)), dict(work=fake(3, 8))):
        assert _scan(L, **kw) == INVALID, kw
    for kw in (dict(x=None), dict(a=None), dict(h=None), dict(work=None)):
        assert _scan(L, **kw) == NULL, kw
    for kw in (dict(n=-1), dict(B=7), dict(D=0), dict(t=-1), dict(s=15), dict(dxs=15), dict(dh=fake(0, 1)), dict(da=fake(0, 1)),
               dict(dl=fake(4, 1)), dict(d0=fake(4, 1)), dict(off=fake(4, 4)), dict(work=fake(3, 8)), dict(dx=fake(0), dxs=20)):
        assert _scan_grad(L, **kw) == INVALID, kw
    for kw in (dict(dh=None), dict(x=None), dict(a=None), dict(h=None), dict(dx=None), dict(da=None), dict(work=None)):
        assert _scan_grad(L, **kw) == NULL, kw
    assert L.gba_recurrence_workspace_size(1, 1, 1, None) == NULL


def test_workspaces_never_fall():
    for D in (1, 16, 64, 511, 4096, 1 << 20):
        for B in (1, 50, 100_000):
            last = last_norm = 0
            for n in sorted({int(1.3 ** k) + d for k in range(80) for d in (-1, 0, 1)}):
                b = gba.gba_recurrence_workspace_size(n, B, D)
                c = gba.gba_residual_norm_grad_workspace_size(n, D)
                assert b >= last and c >= last_norm
                last, last_norm = b, c


def _args(**kw):
    a = gba._ResidualNorm()
    a.n, a.D, a.post, a.pre, a.gate_kind, a.gate_span, a.alpha, a.eps = 12, 16, 2, 2, 1, 4, 1.0, 1e-5
    a.type = a.stream_type = BF16
    for i, k in enumerate(("x", "z", "gate", "h", "y", "post_rstd", "pre_rstd", "dy", "dh", "dx", "dz", "dgate", "dpost_weight",
                           "dpre_weight", "post_weight", "pre_weight")):
        setattr(a, k, fake(i).value)
    for k in ("x", "z", "gate", "h", "y", "dy", "dh", "dx", "dz", "dgate"):
        setattr(a, k + "_stride", kw.get("D", 16))
    for k, v in kw.items():
        setattr(a, k, v.value if isinstance(v, P) else v)
    return a


def _norm(L, **kw):
    for k in ("dy", "dh", "dx", "dz", "dgate", "dpost_weight", "dpre_weight"):
        kw.setdefault(k, None)
    a = _args(**kw)
    return L.gba_residual_norm(ctypes.addressof(a), None)


def _norm_grad(L, ws=1 << 50, work=fake(20), **kw):
    kw.setdefault("y", None)
    a = _args(**kw)
    return L.gba_residual_norm_grad(ctypes.addressof(a), work, SIZE(ws), None)


@no_gpu
@pytest.mark.parametrize("n,D", [(1, 1), (8, 2048), (20_011, 1001), (131_071, 64), (3, 100_003), ((1 << 31) - 1, 8)])
@pytest.mark.parametrize("stream,t", [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)])
def test_residual_norm_host_paths(n, D, stream, t):
    L = gba.lib()
    need = gba.gba_residual_norm_grad_workspace_size(n, D)
    for span in (1, 3, n, 1 << 40):
        s = dict(n=n, D=D, stream_type=stream, type=t, gate_span=span)
        assert _norm(L, **s) == HIP
        assert _norm(L, post=1, pre=1, post_bias=fake(30), pre_bias=fake(31), post_mean=fake(32), pre_mean=fake(33), **s) == HIP
        assert _norm_grad(L, ws=need, **s) == HIP
        assert _norm_grad(L, ws=need - 1, **s) == WORKSPACE
        assert _norm_grad(L, ws=need, gate_kind=0, gate=None, dgate=None, dx=None, dz=None, **s) == HIP
    assert _norm(L, n=0, D=D, x=None, z=None, h=None, y=None, gate=None) == OK


def test_residual_norm_refusals():
    L = gba.lib()
    both = (dict(n=-1), dict(n=1 << 31), dict(D=0), dict(gate_span=0), dict(eps=-1.0), dict(eps=float("nan")), dict(alpha=float("inf")),
            dict(type=3), dict(stream_type=F16), dict(type=F32), dict(weight_type=-1), dict(gate_type=9), dict(post=3), dict(pre=-1),
            dict(gate_kind=3), dict(gate_kind=0), dict(post=0), dict(pre=0), dict(post_bias=fake(30)), dict(pre_bias=fake(30)),
            dict(post_mean=fake(30)), dict(pre_mean=fake(30)), dict(z_stride=15), dict(h_stride=15), dict(gate_stride=15),
            dict(z=fake(1, 1)), dict(h=fake(3, 1)), dict(gate=fake(2, 1)), dict(post_weight=fake(14, 1)), dict(post_rstd=fake(5, 2)))
    for kw in both + (dict(x_stride=15), dict(y=fake(4, 1)), dict(h=fake(0), h_stride=20)):
        assert _norm(L, **kw) == INVALID, kw
    for kw in both + (dict(dy=fake(7, 1)), dict(dh_stride=15), dict(dx=fake(9, 1)), dict(dz_stride=0), dict(dgate_stride=15),
                      dict(dgate=fake(9, 1)), dict(dpost_bias=fake(30)), dict(dpre_weight=fake(13, 2)), dict(grad_type=4),
                      dict(dx=fake(8), dx_stride=20), dict(dz=fake(7), dz_stride=20), dict(work=fake(20, 8))):
        assert _norm_grad(L, **kw) == INVALID, kw
    for kw in (dict(x=None), dict(z=None), dict(h=None), dict(y=None), dict(gate=None)):
        assert _norm(L, **kw) == NULL, kw
    for kw in (dict(z=None), dict(h=None), dict(dy=None), dict(gate=None, dgate=None), dict(post_rstd=None), dict(pre_rstd=None),
               dict(post=1), dict(pre=1), dict(work=None)):
        assert _norm_grad(L, **kw) == NULL, kw
    assert L.gba_residual_norm(None, None) == NULL and L.gba_residual_norm_grad(None, fake(0), SIZE(1 << 50), None) == NULL
    assert L.gba_residual_norm_grad_workspace_size(1, 1, None) == NULL


def _tensors(*given):
    out = (gba._AdamwTensor * max(len(given), 1))()
    for i, kw in enumerate(given):
        t = dict(param=fake(0), grad=fake(1), m=fake(2), v=fake(3), m_exp=None, v_exp=None, copy=None, n=5000, decay=1.0,
                 grad_type=BF16, copy_type=F32, moment_bits=32)
        t.update(kw)
        for k, v in t.items():
            setattr(out[i], k, v.value if isinstance(v, P) else v)
    return out


def _size(*given):
    L, size, chunks = gba.lib(), SIZE(0), ctypes.c_int64(0)
    st = L.gba_adamw_list_size(_tensors(*given), len(given), ctypes.byref(size), ctypes.byref(chunks))
    return st, size.value, chunks.value


def test_adamw_list():
    L = gba.lib()
    assert _size() == (OK, 0, 0)
    st, size, chunks = _size({}, dict(n=0, param=None, grad=None, m=None, v=None), dict(n=1, grad=fake(1, 2)),
                             dict(n=8193, moment_bits=8, m=fake(2, 1), m_exp=fake(4, 3), v_exp=fake(5, 1)))
    assert st == OK and chunks >= 3 and size == 80 * chunks
    t = _tensors({})
    buf = (ctypes.c_char * 4096)()
    st, size, chunks = _size({})
    assert L.gba_adamw_list_fill(t, 1, buf, SIZE(size - 1)) == WORKSPACE
    assert L.gba_adamw_list_fill(t, 1, None, SIZE(size)) == NULL
    assert L.gba_adamw_list_fill(t, 1, buf, SIZE(size)) == OK
    assert L.gba_adamw_list_fill(t, 0, None, SIZE(0)) == OK
    for kw in (dict(n=-1), dict(n=(1 << 40) + 1), dict(grad_type=3), dict(copy_type=-1), dict(moment_bits=16), dict(decay=float("inf")),
               dict(param=fake(0, 2)), dict(grad=fake(1, 1)), dict(m=fake(2, 1)), dict(v=fake(3, 2)), dict(copy=fake(4, 2))):
        assert _size(kw)[0] == INVALID, kw
        assert L.gba_adamw_list_fill(_tensors(kw), 1, buf, SIZE(4096)) == INVALID
    for kw in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(moment_bits=8), dict(moment_bits=8, m_exp=fake(4))):
        assert _size(kw)[0] == NULL, kw
    n = ctypes.c_int64(0)
    assert L.gba_adamw_list_size(None, 1, ctypes.byref(SIZE(0)), ctypes.byref(n)) == NULL
    assert L.gba_adamw_list_size(_tensors(), -1, ctypes.byref(SIZE(0)), ctypes.byref(n)) == INVALID
    assert L.gba_adamw_list_size(_tensors(), (1 << 20) + 1, ctypes.byref(SIZE(0)), ctypes.byref(n)) == INVALID


def _adamw(L, list_=fake(0), chunks=5, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.1, t=1, td=None, coef=None):
    return L.gba_adamw(list_, chunks, lr, b1, b2, eps, wd, t, td, 7, coef, None, None)


@no_gpu
def test_adamw_host_path():
    L = gba.lib()
    assert _adamw(L) == HIP and _adamw(L, td=fake(1), coef=fake(2), b1=0.0, b2=0.0, lr=-1.0, wd=0.0, t=1 << 62) == HIP
    assert _adamw(L, list_=None, chunks=0) == OK


def test_adamw_refusals():
    L = gba.lib()
    for a in ((fake(0), fake(1), -1, 0, fake(2)), (fake(0), fake(1), 5, 2, fake(2)), (fake(0), fake(1), 5, 0, fake(2, 2))):
        assert L.gba_moments_read(*a, None) == INVALID
    assert L.gba_moments_read(None, fake(1), 5, 0, fake(2), None) == NULL and L.gba_moments_read(None, None, 0, 1, None, None) == OK
    for kw in (dict(chunks=-1), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=float("nan")), dict(eps=0.0), dict(eps=1e-45), dict(t=0),
               dict(eps=float("inf")), dict(lr=float("nan")), dict(wd=float("inf")), dict(list_=fake(0, 8)), dict(td=fake(1, 4)), dict(coef=fake(1, 2))):
        assert _adamw(L, **kw) == INVALID, kw
    assert _adamw(L, list_=None) == NULL


# ------------------------------------------------- the float64 forms
def test_the_recurrences_gradient_against_differences():
    rng = np.random.default_rng(1)
    starts, D = np.array([0, 4, 4, 5, 11]), 3
    x, a, dh = (rng.normal(size=(11, D)) for _ in range(3))
    h0, dlast = rng.normal(size=(4, D)), rng.normal(size=(4, D))

    def loss(x, a, h0):
        h, last, _, _ = ref.recurrence(x, a, starts, h0)
        return (h * dh).sum() + (last * dlast).sum()

    h = ref.recurrence(x, a, starts, h0)[0]
    got = ref.recurrence_grad(dh, x, a, h, starts, h0, dlast)[:3]
    for k, g in enumerate(got):
        v, e = rng.normal(size=g.shape), 1e-5
        up, down = [x, a, h0], [x, a, h0]
        up[k], down[k] = up[k] + e * v, down[k] - e * v
        assert abs((loss(*up) - loss(*down)) / (2 * e) - (g * v).sum()) < 1e-7


@pytest.mark.parametrize("mantissa", [3, 4])
def test_codes_stand_for_themselves(mantissa):
    """Every code is its own nearest, whatever is drawn, and the order of codes is that of their values."""
    most = 128 if mantissa == 3 else 256
    code = np.arange(most, dtype=np.uint8)
    if mantissa == 3:
        code = np.concatenate([code, code[1:] + np.uint8(128), [127]]).astype(np.uint8)
    value = ref.decode(code, np.array([130], dtype=np.uint8), mantissa)
    assert (np.diff(value[:most]) > 0).all()
    assert value[:most].max() == (2 - 2.0 ** -mantissa) * 8
    for word in (0, 32768, 65535):
        again, exp = ref.encode(value.astype(np.float32), mantissa, np.full(len(code), word))
        assert exp.tolist() == [130] and np.array_equal(again, code)
