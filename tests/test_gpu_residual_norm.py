"""Norms with gate and residual, and their gradient, against float64.

Tolerances as for the layer norm: u is float32's unit roundoff, an element
passes through no more than D / 64 + 40 additions of a row sum, a sum over n
rows is bounded for any order, and every other operation rounds once; errors are
carried on to first order and widened by a percent.  A sigmoid is off by 6 u of
itself (the exponential 2 u, the sum and the division).  What the second norm
takes is the stream as the call returned it."""
import numpy as np
import pytest
import torch

import paper_2205_11048_amd as gba
from block_reference import BF16, F16, F32, U32, close, gate_factor, matrix, norm_grad, normed, rounded, row_statistics

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-5
NORM = {"none": gba.ROW_NORM_NONE, "layer": gba.ROW_NORM_LAYER, "rms": gba.ROW_NORM_RMS}
GATE = {"none": gba.GATE_NONE, "linear": gba.GATE_LINEAR, "sigmoid": gba.GATE_SIGMOID}


def _ws(n, D):
    return torch.full((gba.gba_residual_norm_grad_workspace_size(n, D),), 255, dtype=torch.uint8, device=DEV)


def _vector(rng, D, dtype, on, mean):
    if not on:
        return None, np.full(D, mean)
    v = torch.from_numpy(mean + 0.3 * rng.normal(size=D)).to(dtype)
    return v.to(DEV), v.double().numpy()


def _statistics_bounds(v64, kind, rstd):
    h = v64.shape[1] / 64 + 40
    dm = 1.01 * (h + 2) * U32 * np.abs(v64).mean(1, keepdims=True) if kind == "layer" else np.zeros((len(v64), 1))
    dr = 1.01 * (0.5 * ((h + 6) * U32 + dm ** 2 * rstd ** 2) + 5 * U32)   # relative
    return dm, dr


def _normed_bound(v64, kind, w, b, mean, rstd):
    if kind == "none":
        return np.zeros_like(v64)
    dm, dr = _statistics_bounds(v64, kind, rstd)
    out = (v64 - mean) * rstd * w + b
    return np.abs(w) * rstd * (dm + np.abs(v64 - mean) * (dr + 4 * U32)) + 2 * U32 * np.abs(out)


class Case:
    def __init__(self, n, D, stream, dtype, wtype=F32, gate="linear", span=1, gtype=F32, post="rms", pre="rms",
                 bias=True, weights=True, alpha=1.0, pad=0, seed=0):
        rng = np.random.default_rng(n * 13 + D + seed)
        self.__dict__.update({k: v for k, v in locals().items() if k not in ("self", "rng")})
        scale = np.exp(rng.normal(size=(n, 1)))
        self.x, self.x64 = matrix(rng.normal(size=(n, D)) * scale, stream, pad)
        self.z, self.z64 = matrix(0.2 + rng.normal(size=(n, D)), dtype, 2 * pad)
        self.rows = np.arange(n) // span
        self.g, self.g64 = matrix(0.3 + rng.normal(size=(-(-n // span), D)), gtype, pad) if gate != "none" else (None, None)
        self.wz, self.wz64 = _vector(rng, D, wtype, weights and post != "none", 1.0)
        self.bz, self.bz64 = _vector(rng, D, wtype, bias and post == "layer", 0.0)
        self.wh, self.wh64 = _vector(rng, D, wtype, weights and pre != "none", 1.0)
        self.bh, self.bh64 = _vector(rng, D, wtype, bias and pre == "layer", 0.0)
        self.dy, self.dy64 = matrix(0.1 * rng.normal(size=(n, D)), dtype, pad)
        self.dh, self.dh64 = matrix(0.1 * rng.normal(size=(n, D)), stream, 2 * pad)
        self.f64, self.df64 = gate_factor(self.g64, gate, self.rows)

    def kw(self):
        return dict(gate=self.g, gate_kind=GATE[self.gate], gate_span=self.span, alpha=self.alpha, eps=EPS,
                    post=NORM[self.post], pre=NORM[self.pre], post_weight=self.wz, post_bias=self.bz,
                    pre_weight=self.wh)

    def new(self, dtype, value=float("nan")):
        return torch.full((self.n, self.D + self.pad), value, dtype=dtype, device=DEV)[:, :self.D]

    def stats(self):
        return {f"{k}_{s}": torch.full((self.n,), float("nan"), device=DEV) for k in ("post", "pre") for s in ("mean", "rstd")
                if getattr(self, k) == "layer" or (getattr(self, k) == "rms" and s == "rstd")}

    def forward(self, h=None, x=None, **stats):
        h = self.new(self.stream) if h is None else h
        y = self.new(self.dtype) if self.pre != "none" else None
        gba.gba_residual_norm(self.x if x is None else x, self.z, h, y, pre_bias=self.bh, **self.kw(), **stats)
        return h, y

    def given_stats(self, h64):
        """The statistics as float32 tensors, and as the values that they then have."""
        t, v = {}, {}
        for name, of in (("post", self.z64), ("pre", h64)):
            kind = getattr(self, name)
            mean, rstd = row_statistics(of, kind, EPS)
            for s, val in (("mean", mean), ("rstd", rstd)):
                if kind == "layer" or (kind == "rms" and s == "rstd"):
                    t[f"{name}_{s}"] = torch.from_numpy(val[:, 0].astype(np.float32)).to(DEV)
                    v[f"{name}_{s}"] = val.astype(np.float32).astype(np.float64)
                else:
                    v[f"{name}_{s}"] = np.zeros_like(val)
        return t, v

    def backward(self, h, stats, dx=None, dz=None, dgate=None, gtype=F32, which="abcd", **kw):
        out = {name: torch.full((self.D,), float("nan"), dtype=gtype, device=DEV)
               for name, k, on in (("dpost_weight", "a", self.post != "none"), ("dpost_bias", "b", self.post == "layer"),
                                   ("dpre_weight", "c", self.pre != "none"), ("dpre_bias", "d", self.pre == "layer"))
               if on and k in which}
        gba.gba_residual_norm_grad(self.dy if self.pre != "none" else None, kw.pop("dh", self.dh), self.z, h, dx, dz,
                                   _ws(self.n, self.D), dgate=dgate, **out, **stats, **self.kw())
        return out


def check_forward(c):
    stats = c.stats()
    h, y = c.forward(**stats)
    mean, rstd = row_statistics(c.z64, c.post, EPS)
    u = normed(c.z64, c.post, c.wz64, c.bz64, EPS)
    ref = c.alpha * c.x64 + c.f64 * u
    bound = np.abs(c.f64) * (_normed_bound(c.z64, c.post, c.wz64, c.bz64, mean, rstd) + 7 * U32 * np.abs(u))
    bound = bound + 3 * U32 * np.abs(c.alpha * c.x64) + U32 * np.abs(ref)
    close(h, ref, rounded(bound, ref, c.stream), "h")
    h64 = h.double().cpu().numpy()
    for name, kind, v in (("post", c.post, c.z64), ("pre", c.pre, h64)):
        if kind == "none":
            continue
        m, r = row_statistics(v, kind, EPS)
        dm, dr = _statistics_bounds(v, kind, r)
        close(stats[name + "_rstd"], r[:, 0], (dr * r)[:, 0], name + "_rstd")
        if kind == "layer":
            close(stats[name + "_mean"], m[:, 0], dm[:, 0] + 1e-38, name + "_mean")
    if c.pre != "none":
        m, r = row_statistics(h64, c.pre, EPS)
        ref = normed(h64, c.pre, c.wh64, c.bh64, EPS)
        close(y, ref, rounded(_normed_bound(h64, c.pre, c.wh64, c.bh64, m, r), ref, c.dtype), "y")
    # without the statistics, the stream in place: the same bits
    x = c.x.clone() if not c.pad else torch.empty((c.n, c.D + c.pad), dtype=c.stream, device=DEV)[:, :c.D].copy_(c.x)
    _, y2 = c.forward(h=x, x=x)
    assert torch.equal(x, h) and (y is None or torch.equal(y2, y))
    for t in (h, y):
        if t is not None and c.pad:
            assert torch.isnan(t.as_strided((c.n, c.D + c.pad), t.stride())[:, c.D:]).all()
    return h, h64


def check_backward(c, h, h64):
    n, D, hd = c.n, c.D, c.D / 64 + 40
    stats, v = c.given_stats(h64)
    dx, dz = c.new(c.stream), c.new(c.dtype)
    dg = torch.full_like(c.g, float("nan")) if c.g is not None else None
    out = c.backward(h, stats, dx, dz, dg)
    # the stream's gradient
    pre, xh = norm_grad(c.dy64, h64, c.pre, c.wh64, v["pre_mean"], v["pre_rstd"])
    e, Be = c.dh64, np.zeros((n, D))
    if c.pre != "none":
        hh, r = c.dy64 * c.wh64, v["pre_rstd"]
        s1 = hh.mean(1, keepdims=True) * (c.pre == "layer")
        s2 = (hh * xh).mean(1, keepdims=True)
        d1 = (hd + 4) * U32 * np.abs(hh).mean(1, keepdims=True)
        d2 = (hd + 8) * U32 * np.abs(hh * xh).mean(1, keepdims=True)
        Be = r * (6 * U32 * (np.abs(hh) + np.abs(s1) + 2 * np.abs(xh * s2)) + d1 + np.abs(xh) * d2)
        Be = Be + 2 * U32 * (np.abs(c.dh64) + np.abs(pre))
        e = c.dh64 + pre
        each = c.dy64 * xh
        close(out["dpre_weight"], each.sum(0), 1.01 * (n + 8) * U32 * np.abs(each).sum(0) + 1e-38, "dpre_weight")
        if c.pre == "layer":
            close(out["dpre_bias"], c.dy64.sum(0), 1.01 * (n + 4) * U32 * np.abs(c.dy64).sum(0) + 1e-38, "dpre_bias")
    ref = c.alpha * e
    close(dx, ref, rounded(abs(c.alpha) * Be + 3 * U32 * np.abs(ref), ref, c.stream), "dx")
    # the block's
    zh = (c.z64 - v["post_mean"]) * v["post_rstd"] if c.post != "none" else c.z64
    u = zh * c.wz64 + c.bz64
    Bu = 4 * U32 * np.abs(zh * c.wz64) + U32 * np.abs(u)
    k = e * c.f64
    Bk = np.abs(c.f64) * Be + 7 * U32 * np.abs(k)
    if c.gate != "none":
        df_err = 7 * U32 * np.abs(c.df64)
        if c.gate == "sigmoid":
            df_err = df_err + c.f64 * (6 * U32 * c.f64 + U32)
        each = e * u * c.df64
        B = np.abs(u * c.df64) * Be + np.abs(e * c.df64) * Bu + np.abs(e * u) * df_err + 3 * U32 * np.abs(each)
        G = c.g64.shape[0]
        ref, bound, size, count = (np.zeros((G, D)) for _ in range(4))
        # (rows that share a gate add up e * zh and e apart: their sum is w * one + b * the other, whose terms are these)
        terms = np.abs(e * c.df64) * (np.abs(zh * c.wz64) + np.abs(c.bz64)) if c.span > 1 else np.abs(each)
        for to, val in ((ref, each), (bound, B), (size, terms), (count, np.ones_like(each))):
            np.add.at(to, c.rows, val)
        close(dg, ref, rounded(bound + (count + 4) * U32 * size * (c.span > 1), ref, c.gtype), "dgate")
    if c.post == "none":
        ref, bound = k, Bk
    else:
        each = k * zh
        close(out["dpost_weight"], each.sum(0),
              1.01 * ((Bk * np.abs(zh)).sum(0) + (n + 8) * U32 * np.abs(each).sum(0)) + 1e-38, "dpost_weight")
        if c.post == "layer":
            close(out["dpost_bias"], k.sum(0), 1.01 * (Bk.sum(0) + (n + 4) * U32 * np.abs(k).sum(0)) + 1e-38, "dpost_bias")
        kk, r = k * c.wz64, v["post_rstd"]
        Bkk = Bk * np.abs(c.wz64) + U32 * np.abs(kk)
        m1 = kk.mean(1, keepdims=True) * (c.post == "layer")
        m2 = (kk * zh).mean(1, keepdims=True)
        d1 = (hd + 4) * U32 * np.abs(kk).mean(1, keepdims=True) + Bkk.mean(1, keepdims=True)
        d2 = (hd + 8) * U32 * np.abs(kk * zh).mean(1, keepdims=True) + (Bkk * np.abs(zh)).mean(1, keepdims=True)
        ref = r * (kk - m1 - zh * m2)
        bound = r * (Bkk + 6 * U32 * (np.abs(kk) + np.abs(m1) + 2 * np.abs(zh * m2)) + d1 + np.abs(zh) * d2)
    close(dz, ref, rounded(bound, ref, c.dtype), "dz")
    for t in (dx, dz):
        if c.pad:
            assert torch.isnan(t.as_strided((n, D + c.pad), t.stride())[:, D:]).all()
    # each alone, the parameters' in another type, and in place: the same bits
    for which in "abcd":
        for name, t in c.backward(h, stats, which=which).items():
            assert torch.equal(t, out[name]), name
    for name, t in c.backward(h, stats, gtype=BF16).items():
        assert torch.equal(t, out[name].to(BF16)), name
    if dg is not None:
        dg2 = torch.full_like(dg, float("nan"))
        c.backward(h, stats, dgate=dg2, which="")
        assert torch.equal(dg2, dg)
    out2 = c.backward(h, stats, dx=c.dh, dz=c.dy if c.pre != "none" else None)
    assert torch.equal(c.dh, dx) and (c.pre == "none" or torch.equal(c.dy, dz))
    assert all(torch.equal(out2[k], out[k]) for k in out)


def check(*args, **kw):
    c = Case(*args, **kw)
    check_backward(c, *check_forward(c))


SIZES = [(1, 1), (3, 2), (1, 8), (7, 16), (129, 31), (300, 32), (257, 64), (65, 100), (40, 255), (64, 257), (33, 520),
         (8, 1024), (41, 1001), (1, 2048), (70, 2048), (37, 4096), (11, 4100), (9, 8192), (5, 10_007)]


@pytest.mark.parametrize("n,D", SIZES)
def test_sizes_in_32_bits(n, D):
    check(n, D, F32, F32, gate="sigmoid", span=1, post="layer", pre="layer", alpha=0.8, pad=3 if D % 2 else 0)


@pytest.mark.parametrize("n,D", SIZES)
def test_sizes_in_16_bits(n, D):
    check(n, D, BF16, BF16, wtype=BF16, gate="linear", span=max(n // 3, 1), gtype=BF16)


@pytest.mark.parametrize("stream,dtype", [(F32, BF16), (F32, F16), (F16, F16)])
@pytest.mark.parametrize("n,D", [(3, 5), (130, 48), (33, 600), (9, 2048), (5, 5000)])
def test_types(n, D, stream, dtype):
    check(n, D, stream, dtype, wtype=dtype, gate="linear", span=n, gtype=dtype, post="rms", pre="layer", pad=1)


@pytest.mark.parametrize("gate", ["none", "linear", "sigmoid"])
@pytest.mark.parametrize("post,pre", [("none", "none"), ("none", "rms"), ("none", "layer"), ("rms", "none"),
                                      ("layer", "none"), ("rms", "layer"), ("layer", "rms")])
def test_norms_and_gates(post, pre, gate):
    for n, D in ((50, 136), (6, 3000)):
        check(n, D, F32, F32, gate=gate, span=7, post=post, pre=pre, alpha=-1.3)
        check(n, D, F32, BF16, gate=gate, span=1, post=post, pre=pre, weights=False, bias=False)


@pytest.mark.parametrize("n,D,span", [(1000, 24, 1), (1000, 24, 2), (1000, 24, 3), (1025, 40, 500), (1025, 40, 1024),
                                      (1025, 40, 1025), (1025, 40, 1 << 40), (3000, 8, 5), (777, 130, 64), (600, 520, 150),
                                      (1100, 600, 1)])
def test_rows_that_share_a_gate(n, D, span):
    check(n, D, F32, F32, gate="linear", span=span)
    check(n, D, BF16, BF16, gate="sigmoid", span=span, gtype=BF16, post="layer")


@pytest.mark.parametrize("n,D,span", [(2501, 8, 2), (4801, 24, 3), (2100, 130, 2), (4700, 300, 3), (2200, 2, 2), (40_000, 16, 8)])
def test_many_gates_of_few_rows(n, D, span):
    """A gate row for each group of lanes (more than 512 times as many as rows share one)."""
    check(n, D, F32, F32, gate="linear", span=span, post="layer", pre="rms")
    check(n, D, F32, BF16, gate="sigmoid", span=span, gtype=BF16, post="rms", pre="layer")
    check(n, D, BF16, BF16, gate="linear", span=span, gtype=F32, post="none", pre="none")


def test_many_rows():
    check(9001, 40, F32, F32, gate="linear", span=9001, post="layer", pre="layer")
    check(5003, 264, BF16, BF16, gate="sigmoid", span=1)


def test_no_gradient_from_elsewhere():
    c = Case(30, 80, F32, F32)
    h, h64 = check_forward(c)
    stats, _ = c.given_stats(h64)
    zero = torch.zeros_like(c.dh)
    outs = []
    for dh in (None, zero):
        dx, dz = c.new(F32), c.new(F32)
        outs.append((dx, dz, *c.backward(h, stats, dx, dz, dh=dh).values()))
    assert all(torch.equal(p, q) for p, q in zip(*outs))


def test_the_gradient_is_the_forwards():
    """Central differences in float64 of L = sum(c * y) + sum(d * h), in every argument: at a step of 1e-5 they leave
    out 1e-10 of the third derivatives, and the kernel is off by its bounds, 100 u of sums of a few magnitudes."""
    c = Case(6, 20, F32, F32, gate="sigmoid", span=4, post="layer", pre="layer", alpha=0.7, seed=5)
    h, h64 = check_forward(c)
    stats, _ = c.given_stats(h64)
    dx, dz, dg = c.new(F32), c.new(F32), torch.empty_like(c.g)
    out = c.backward(h, stats, dx, dz, dg)

    def loss(p):
        u = normed(p["z"], "layer", p["wz"], p["bz"], EPS)
        s = p["alpha"] * p["x"] + gate_factor(p["g"], "sigmoid", c.rows)[0] * u
        return (normed(s, "layer", p["wh"], p["bh"], EPS) * c.dy64).sum() + (s * c.dh64).sum()

    at = dict(x=c.x64, z=c.z64, g=c.g64, wz=c.wz64, bz=c.bz64, wh=c.wh64, bh=c.bh64, alpha=c.alpha)
    got = dict(x=dx, z=dz, g=dg, wz=out["dpost_weight"], bz=out["dpost_bias"], wh=out["dpre_weight"],
               bh=out["dpre_bias"])
    rng = np.random.default_rng(3)
    for name, t in got.items():
        g = t.double().cpu().numpy()
        v = rng.normal(size=g.shape)
        e = 1e-5
        quotient = (loss({**at, name: at[name] + e * v}) - loss({**at, name: at[name] - e * v})) / (2 * e)
        # (the stream that the second norm takes is rounded: u of it more)
        assert abs(quotient - (g * v).sum()) <= 200 * U32 * np.abs(g * v).sum() + 200 * U32 * np.abs(v).sum(), name


def test_no_rows():
    D = 24
    x = torch.empty((0, D), device=DEV)
    w = torch.ones(D, device=DEV)
    gba.gba_residual_norm(x, x, x, x, post_weight=w, pre_weight=w)
    outs = [torch.full((D,), 5.0, device=DEV) for _ in range(2)]
    none = torch.empty(0, device=DEV)
    gba.gba_residual_norm_grad(x, x, x, x, x, x, _ws(0, D), post_weight=w, pre_weight=w, post_rstd=none, pre_rstd=none,
                               dpost_weight=outs[0], dpre_weight=outs[1])
    assert all((t == 0).all() for t in outs)


@pytest.mark.parametrize("D", [96, 9000])
def test_rows_keep_their_infinities(D):
    x, z = torch.ones((5, D), device=DEV), torch.randn((5, D), device=DEV)
    x[1, 5], z[3, 6] = float("inf"), float("nan")
    z[4] = 0.0   # a row of nothing
    w = torch.ones(D, device=DEV)
    h, y = torch.empty_like(x), torch.empty_like(x)
    gba.gba_residual_norm(x, z, h, y, post_weight=w, pre_weight=w)
    assert torch.isfinite(y[[0, 2, 4]]).all() and not torch.isfinite(y[1]).all() and torch.isnan(y[3]).all()
    assert (h[4] == 1.0).all()


def test_in_a_graph_and_on_another_stream():
    c = Case(700, 264, BF16, BF16, gate="linear", span=100, gtype=BF16)
    stats = c.stats()
    h, y = c.forward(**stats)
    dx, dz, dg = c.new(BF16), c.new(BF16), torch.empty_like(c.g)
    ws = _ws(c.n, c.D)
    dw = [torch.empty(c.D, device=DEV) for _ in range(2)]

    def both(**kw):
        gba.gba_residual_norm(c.x, c.z, h, y, **c.kw(), **stats, **kw)
        gba.gba_residual_norm_grad(c.dy, c.dh, c.z, h, dx, dz, ws, dgate=dg, dpost_weight=dw[0], dpre_weight=dw[1],
                                   **c.kw(), **stats, **kw)

    outs = (h, y, dx, dz, dg, *dw, *stats.values())
    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    other = torch.cuda.Stream()
    for t in outs:
        t.fill_(float("nan"))
    torch.cuda.synchronize()
    both(stream=other)
    other.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(4):
        c.x.neg_()
        c.z.neg_()
        for t in outs:
            t.fill_(float("nan"))
        ws.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        if k % 2:
            assert all(torch.equal(p, q) for p, q in zip(outs, want))
        else:   # (the block's output and the stream turned round: so are h and y)
            assert torch.equal(h, -want[0]) and torch.equal(y, -want[1])


def test_refusals():
    x, w, g = torch.zeros((6, 16), device=DEV), torch.ones(16, device=DEV), torch.ones((2, 16), device=DEV)
    s, ws = torch.zeros(6, device=DEV), _ws(6, 16)
    f, b = gba.gba_residual_norm, gba.gba_residual_norm_grad
    NONE, LAYER = gba.ROW_NORM_NONE, gba.ROW_NORM_LAYER
    for bad in [lambda: f(x, x, x.half(), x), lambda: f(x.half(), x, x.half(), x), lambda: f(x[:5], x, x, x), lambda: f(x, x, x),   # (z says how many rows there are)
               
                lambda: f(x, x, x, x, pre=NONE), lambda: f(x, x, x, x, gate=g, gate_span=2), lambda: f(x, x, x, x, gate=g, gate_span=0),
                lambda: f(x, x, x, x, gate_kind=gba.GATE_SIGMOID), lambda: f(x, x, x, x, gate=g, gate_span=3, gate_kind=gba.GATE_NONE),
                lambda: f(x, x, x, x, post=3), lambda: f(x, x, x, x, post_bias=w), lambda: f(x, x, x, x, post=NONE, post_weight=w),
                lambda: f(x, x, x, x, post=NONE, post_rstd=s), lambda: f(x, x, x, x, pre_mean=s), lambda: f(x, x, x, x, eps=-1.0),
                lambda: f(x, x, x, x, eps=float("nan")), lambda: f(x, x, x, x, alpha=float("inf")), lambda: f(x, x, x, x, post_weight=w[:15]),
                lambda: f(x, x, x, x, post_weight=w, pre_weight=w.half()), lambda: f(x, x, x, x, pre_rstd=s[:5]), lambda: f(x.cpu(), x, x, x),
                lambda: f(x.T, x.T, x.T, x.T),
                lambda: b(x, x, x, x, x, x, ws[:-1], post_rstd=s, pre_rstd=s), lambda: b(x, x, x, x, x, x, ws, pre_rstd=s),
                lambda: b(None, x, x, x, x, x, ws, post_rstd=s, pre_rstd=s), lambda: b(x, x, x, None, x, x, ws, post_rstd=s, pre_rstd=s),
                lambda: b(x, x, x, x, x, x, ws, post=LAYER, post_rstd=s, pre_rstd=s), lambda: b(x, x.half(), x, x, x, x, ws, post_rstd=s, pre_rstd=s),
                lambda: b(x, x, x, x, x, x, ws, post_rstd=s, pre_rstd=s, dpre_bias=w), lambda: b(x, x, x, x, x, x, ws, post_rstd=s, pre_rstd=s, dgate=g),
                lambda: b(x, x, x, x, x, x, ws, gate=g, gate_span=3, post_rstd=s, pre_rstd=s, dgate=g.half()),
                lambda: b(x, x, x, x, x, x, ws, post=NONE, pre_rstd=s, dpost_weight=w),
                lambda: gba.gba_residual_norm_grad_workspace_size(-1, 16), lambda: gba.gba_residual_norm_grad_workspace_size(5, 0)]:
        with pytest.raises(gba.GBAError):
            bad()


def test_rows_far_apart_and_many():
    """Strides of 2^22 elements (more than 2^32 bytes from the first row to the last), and more than 2^31 elements."""
    n, D = 600, 96
    far = torch.empty(n << 22, dtype=BF16, device=DEV).as_strided((n, D), (1 << 22, 1))
    x, z = torch.randn((n, D), device=DEV).to(BF16), torch.randn((n, D), device=DEV).to(BF16)
    want, got = [torch.empty_like(x) for _ in range(2)], [torch.empty_like(x) for _ in range(2)]
    gba.gba_residual_norm(x, z, *want)
    far.copy_(z)
    gba.gba_residual_norm(x, far, *got)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    far.copy_(x)
    gba.gba_residual_norm(far, z, far, got[1])
    assert torch.equal(far, want[0]) and torch.equal(got[1], want[1])
    stats = dict(post_rstd=torch.rand(n, device=DEV), pre_rstd=torch.rand(n, device=DEV))
    grads = [[torch.empty_like(x) for _ in range(2)] for _ in range(2)]
    gba.gba_residual_norm_grad(x, x, z, want[0], *grads[0], _ws(n, D), **stats)
    far.copy_(want[0])
    gba.gba_residual_norm_grad(x, x, z, far, *grads[1], _ws(n, D), **stats)
    assert all(torch.equal(p, q) for p, q in zip(*grads))
    del far
    n = (1 << 25) + 3
    x, z = x[:1].expand(n, D).contiguous(), z[:1].expand(n, D).contiguous()
    h, y = torch.empty_like(x), torch.empty_like(x)
    gba.gba_residual_norm(x, z, h, y)
    assert (h == want[0][0]).all() and (y == want[1][0]).all()
    stats = dict(post_rstd=torch.ones(n, device=DEV), pre_rstd=torch.ones(n, device=DEV))
    gba.gba_residual_norm_grad(y, z, z, h, x, y, _ws(n, D), **stats)
    assert (x == x[0]).all() and (y == y[0]).all()
