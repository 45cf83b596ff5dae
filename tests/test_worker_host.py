"""Host paths of the worker's operators on a machine without a GPU: argument
checks, size queries, the tensor list, and each call with fake device addresses
up to its first launch, which fails because there is no device."""
import ctypes

import pytest

import paper_2205_11048_amd as gba


def _gpu_visible():
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:
        return False


no_gpu = pytest.mark.skipif(_gpu_visible(), reason="fake device addresses must never reach a GPU")

OK, NULL, INVALID, WORKSPACE, HIP = 0, 1, 2, 4, 5
P, SIZE = ctypes.c_void_p, ctypes.c_size_t
F32, BF16, F16 = 0, 1, 2


def fake(i, offset=0):
    return P((1 << 20) * (i + 1) + offset)


def _lookup(L, n=5, R=100, D=16, t=F32, ts=16, o=F32, os=16, ids=fake(0), table=fake(1), out=fake(2), width=8):
    return L.gba_embedding_lookup(ids, width, n, table, t, ts, R, D, 1.0, out, o, os, None, None)


@no_gpu
def test_lookup_host_path():
    L = gba.lib()
    assert _lookup(L) == HIP
    assert _lookup(L, n=0, ids=None, table=None, out=None) == OK
    assert _lookup(L, n=(1 << 31) - 1, R=1 << 32, D=1 << 20, ts=1 << 20, os=1 << 40) == HIP
    assert _lookup(L, table=fake(1, 2), t=BF16) == HIP          # an element's alignment is enough
    assert _lookup(L, ids=fake(0, 4), width=4) == HIP


def test_lookup_refusals():
    L = gba.lib()
    for kw in (dict(n=-1), dict(n=1 << 31), dict(R=0), dict(R=(1 << 32) + 1), dict(D=0), dict(D=(1 << 20) + 1, ts=1 << 21),
               dict(ts=15), dict(os=15), dict(t=3), dict(o=-1), dict(table=fake(1, 2)), dict(out=fake(2, 1), o=BF16),
               dict(ids=fake(0, 4)), dict(ids=fake(0, 2), width=4), dict(width=2), dict(width=16)):
        assert _lookup(L, **kw) == INVALID, kw
    for kw in (dict(ids=None), dict(table=None), dict(out=None)):
        assert _lookup(L, **kw) == NULL, kw


SIZES = [(1, 1, 1), (130, 8, 7), (16_384, 4096, 100_000), (256_000, 32, 100_000_000), ((1 << 28) - 1, 1 << 20, 1 << 32)]


def _rows(L, n, D, R, ws, **kw):
    a = dict(ids=fake(0), grad=fake(1), g=BF16, gs=D, unique=fake(2), rows=fake(3), rs=D, num=fake(4), work=fake(5))
    a.update(kw)
    return L.gba_embedding_grad_rows(a["ids"], n, a["grad"], a["g"], a["gs"], D, R, 1.0, -1, a["unique"], a["rows"], a["rs"],
                                     a["num"], a["work"], SIZE(ws), None, None)


def _dense(L, n, D, R, ws, **kw):
    a = dict(ids=fake(0), grad=fake(1), g=BF16, gs=D, table=fake(2), o=F32, os=D, work=fake(5))
    a.update(kw)
    return L.gba_embedding_grad_dense(a["ids"], n, a["grad"], a["g"], a["gs"], D, R, 1.0, -1, a["table"], a["o"], a["os"], 0,
                                      a["work"], SIZE(ws), None, None)


@no_gpu
@pytest.mark.parametrize("n,D,R", SIZES)
def test_embedding_grad_host_paths(n, D, R):
    L = gba.lib()
    need = gba.gba_embedding_grad_workspace_size(n, D, R)
    for call in (_rows, _dense):
        assert call(L, n, D, R, need - 1) == WORKSPACE
        assert call(L, n, D, R, need) == HIP


def test_embedding_grad_refusals():
    L = gba.lib()
    ws = 1 << 40
    for kw in (dict(g=3), dict(gs=7), dict(ids=fake(0, 8)), dict(work=fake(5, 8)), dict(grad=fake(1, 1))):
        assert _rows(L, 10, 8, 100, ws, **kw) == INVALID, kw
        assert _dense(L, 10, 8, 100, ws, **kw) == INVALID, kw
    for kw in (dict(ids=None), dict(grad=None), dict(work=None)):
        assert _rows(L, 10, 8, 100, ws, **kw) == NULL, kw
        assert _dense(L, 10, 8, 100, ws, **kw) == NULL, kw
    for n, D, R in [(-1, 8, 100), (1 << 28, 8, 100), (10, 0, 100), (10, 8, 0), (10, 8, (1 << 32) + 1)]:
        assert _rows(L, n, D, R, ws, gs=64, rs=64) == INVALID
        assert _dense(L, n, D, R, ws, gs=64, os=64) == INVALID
    assert _rows(L, 10, 8, 100, ws, rs=7) == INVALID and _rows(L, 10, 8, 100, ws, rows=fake(3, 2)) == INVALID
    assert _dense(L, 10, 8, 100, ws, os=7) == INVALID and _dense(L, 10, 8, 100, ws, o=9) == INVALID
    for kw in (dict(unique=None), dict(rows=None), dict(num=None)):
        assert _rows(L, 10, 8, 100, ws, **kw) == NULL
    assert _dense(L, 10, 8, 100, ws, table=None) == NULL


@pytest.mark.parametrize("D,R", [(1, 5), (8, 1 << 20), (32, 100_000_000), (100, 50_000), (4096, 100_000)])
def test_workspaces_never_fall(D, R):
    """Scratch for the largest input serves every smaller one."""
    sizes = sorted({int(1.17 ** k) + d for k in range(120) for d in (-1, 0, 1) if 0 <= int(1.17 ** k) + d < 1 << 28})
    last = last_ln = 0
    for n in sizes:
        b, c = gba.gba_embedding_grad_workspace_size(n, D, R), gba.gba_layer_norm_grad_workspace_size(n, D)
        assert b >= last and c >= last_ln, n
        last, last_ln = b, c


def _norm(L, n=4, D=16, t=BF16, w=F32, x=fake(0), xs=16, y=fake(1), ys=16, weight=fake(2), bias=fake(3), eps=1e-5):
    return L.gba_layer_norm(x, xs, t, n, D, weight, bias, w, eps, y, ys, fake(4), None, None)


def _norm_grad(L, n=4, D=16, t=BF16, w=F32, g=F32, dy=fake(0), dys=16, x=fake(1), xs=16, mean=fake(2), rstd=fake(3),
               weight=fake(4), dx=fake(5), dxs=16, dw=fake(6), db=fake(7), work=fake(8), ws=None):
    ws = gba.gba_layer_norm_grad_workspace_size(min(max(n, 0), (1 << 31) - 1), min(max(D, 1), 1 << 20)) if ws is None else ws
    return L.gba_layer_norm_grad(dy, dys, x, xs, t, n, D, mean, rstd, weight, w, dx, dxs, dw, db, g, work, SIZE(ws), None)


@no_gpu
@pytest.mark.parametrize("n,D", [(1, 1), (8, 2048), (20_011, 1001), (256_000, 64), (3, 100_003), ((1 << 31) - 1, 8)])
@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_layer_norm_host_paths(n, D, t):
    L = gba.lib()
    s = dict(xs=D, ys=D)
    assert _norm(L, n, D, t, **s) == HIP
    assert _norm(L, n, D, t, weight=None, bias=None, **s) == HIP
    s = dict(xs=D, dys=D, dxs=D)
    assert _norm_grad(L, n, D, t, **s) == HIP
    assert _norm_grad(L, n, D, t, dx=None, weight=None, **s) == HIP
    assert _norm_grad(L, n, D, t, dw=None, db=None, **s) == HIP
    need = gba.gba_layer_norm_grad_workspace_size(n, D)
    assert _norm_grad(L, n, D, t, ws=need - 1, **s) == WORKSPACE


def test_layer_norm_refusals():
    L = gba.lib()
    for kw in (dict(n=-1), dict(D=0), dict(t=4), dict(w=4), dict(xs=15), dict(ys=15), dict(eps=-1.0),
               dict(eps=float("nan")), dict(x=fake(0, 1)), dict(weight=fake(2, 2)), dict(bias=fake(3, 1)),
               dict(y=fake(0), ys=17)):
        assert _norm(L, **kw) == INVALID, kw
    assert _norm(L, x=None) == NULL and _norm(L, y=None) == NULL
    assert _norm(L, n=0, x=None, y=None) == OK
    for kw in (dict(n=-1), dict(D=0), dict(t=-1), dict(w=3), dict(g=3), dict(dys=1), dict(xs=1), dict(dxs=1),
               dict(dx=fake(0), dxs=17), dict(work=fake(8, 4)), dict(dw=fake(6, 2)), dict(db=fake(7, 1))):
        assert _norm_grad(L, **kw) == INVALID, kw
    for kw in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(work=None)):
        assert _norm_grad(L, **kw) == NULL, kw


def _tensors(*entries):
    return (gba._Tensor * len(entries))(*[gba._Tensor(*e) for e in entries])


def test_tensor_list():
    L = gba.lib()
    size, chunks = SIZE(0), ctypes.c_int64(0)
    t = _tensors((1 << 20, 2 << 20, None, 100_000, 1, F32, BF16), (3 << 20, None, None, 0, 1, F16, F16),
                 (4 << 20, 4 << 20, 5 << 20, 640, 64, F32, F32))
    assert L.gba_tensor_list_size(t, 3, ctypes.byref(size), ctypes.byref(chunks)) == OK
    assert chunks.value >= 2 and size.value % chunks.value == 0
    image = ctypes.create_string_buffer(size.value + 16)
    assert L.gba_tensor_list_fill(t, 3, image, SIZE(size.value)) == OK
    assert image.raw[size.value:] == b"\0" * 16
    assert L.gba_tensor_list_fill(t, 3, image, SIZE(size.value - 1)) == WORKSPACE
    assert L.gba_tensor_list_fill(t, 3, None, SIZE(size.value)) == NULL
    assert L.gba_tensor_list_size(None, 0, ctypes.byref(size), ctypes.byref(chunks)) == OK
    assert (size.value, chunks.value) == (0, 0)
    assert L.gba_tensor_list_fill(None, 0, None, SIZE(0)) == OK


def test_tensor_list_refusals():
    L = gba.lib()
    size, chunks = SIZE(0), ctypes.c_int64(0)
    A = 1 << 20
    for e in ((A, None, None, -1, 1, F32, F32), (A, None, None, (1 << 40) + 1, 1, F32, F32), (A, None, None, 5, 1, 3, F32),
              (A, None, None, 5, 1, F32, -1), (A + 2, None, None, 5, 1, F32, F32), (A, A + 1, None, 5, 1, F32, BF16),
              (A, A, None, 5, 1, F32, BF16), (A, None, A, 5, 0, F32, F32)):
        t = _tensors(e)
        assert L.gba_tensor_list_size(t, 1, ctypes.byref(size), ctypes.byref(chunks)) == INVALID, e
        assert L.gba_tensor_list_fill(t, 1, None, SIZE(0)) == INVALID, e
    t = _tensors((None, None, None, 5, 1, F32, F32))
    assert L.gba_tensor_list_size(t, 1, ctypes.byref(size), ctypes.byref(chunks)) == NULL
    assert L.gba_tensor_list_size(None, 1, ctypes.byref(size), ctypes.byref(chunks)) == NULL
    assert L.gba_tensor_list_size(t, -1, ctypes.byref(size), ctypes.byref(chunks)) == INVALID
    assert L.gba_tensor_list_size(t, 1, None, ctypes.byref(chunks)) == NULL


def test_clip_refusals():
    L = gba.lib()

    def clip(chunks=3, max_norm=1.0, lst=fake(0), norm=fake(1), work=fake(2), ws=1 << 20):
        return L.gba_clip_grads(lst, chunks, max_norm, norm, None, work, SIZE(ws), None, None)

    for kw in (dict(chunks=-1), dict(max_norm=0.0), dict(max_norm=-2.0), dict(max_norm=float("nan")),
               dict(work=fake(2, 8)), dict(lst=fake(0, 8))):
        assert clip(**kw) == INVALID, kw
    for kw in (dict(lst=None), dict(norm=None), dict(work=None)):
        assert clip(**kw) == NULL, kw
    assert clip(ws=8) == WORKSPACE
    assert L.gba_grad_norm(None, 3, fake(1), fake(2), SIZE(1 << 20), None, None) == NULL
    assert L.gba_grad_norm(fake(0), 3, fake(1), fake(2), SIZE(0), None, None) == WORKSPACE
    if not _gpu_visible():
        assert clip() == HIP and clip(chunks=0, lst=None) == HIP
        assert L.gba_grad_norm(fake(0), 1 << 30, fake(1), fake(2), SIZE(1 << 20), None, None) == HIP
