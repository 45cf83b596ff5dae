"""The worker's sequence block and optimiser as measurable cases.

Each case is one pass through one operator of ``paper_2205_11048_amd``:

* ``norm_fwd``, ``norm_bwd``   -- a block's output normalised, gated and added to the scaled residual
                                  stream, and the stream normalised for the next block; its gradient;
* ``scan_fwd``, ``scan_bwd``   -- a gated linear recurrence over the positions of many sequences (one
                                  position each while serving) and its gradient;
* ``adamw``                    -- one AdamW step over many tensors, with the moments in 32 or in 8 bits.

With ``own`` false the operators run in their plain form, elementary torch operations in 32 bits; with
``own`` true through the library.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
SIGMA = 1e-2         # standard deviation of the gradients
DEV = "cuda"
LR, BETA1, BETA2, ADAM_EPS, DECAY, SEED = 1e-3, 0.9, 0.999, 1e-8, 0.01, 2_718_281
BLOCK = 256          # values of an 8-bit moment that share an exponent


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # a decoding step of eight sequences, the gate one scale a channel: latency only
        dict(name="norm_fwd_decode", op="norm_fwd", n=8, D=2_048, stream="bf16", type="bf16", wtype="bf16",
             gate="linear", span=8, gtype="bf16", post="rms", pre="rms", bias=0, alpha=1.0, pad=0),
        # a training batch of 16 sequences of 1024 tokens, a gate for each sequence
        dict(name="norm_fwd_train", op="norm_fwd", n=16_384, D=4_096, stream="bf16", type="bf16", wtype="bf16",
             gate="linear", span=1_024, gtype="bf16", post="rms", pre="rms", bias=0, alpha=1.0, pad=0),
        # its backward pass
        dict(name="norm_bwd_train", op="norm_bwd", n=16_384, D=4_096, stream="bf16", type="bf16", wtype="f32",
             gate="linear", span=1_024, gtype="bf16", post="rms", pre="rms", bias=0, alpha=1.0, pad=0),
        # narrow rows of a recommender's activations, a gate for each token, layer norms with biases, inside wider
        # tensors
        dict(name="norm_bwd_narrow", op="norm_bwd", n=131_071, D=64, stream="f32", type="f32", wtype="f32",
             gate="sigmoid", span=1, gtype="f32", post="layer", pre="layer", bias=1, alpha=0.8, pad=8),
        # one new token of 64 sequences, the states updated: latency only
        dict(name="scan_step", op="scan_fwd", B=64, L=1, n=64, D=2_048, type="bf16", state=1, tail=0, pad=0),
        # a training batch of 32 sequences of 1024 tokens
        dict(name="scan_train", op="scan_fwd", B=32, L=1_024, n=32_768, D=2_048, type="bf16", state=0, tail=0, pad=0),
        # behaviour histories of users, packed: ragged, some empty, narrow rows, room behind the last
        dict(name="scan_histories", op="scan_fwd", B=4_096, L=0, n=205_000, D=64, type="f32", state=1, tail=777,
             pad=0),
        # the backward pass of a training batch
        dict(name="scan_bwd_train", op="scan_bwd", B=16, L=2_048, n=32_768, D=2_048, type="bf16", state=0, tail=0,
             pad=0),
        # the backward pass over one long sequence of an odd width, with gradients of its last and first states
        dict(name="scan_bwd_long", op="scan_bwd", B=1, L=100_003, n=100_003, D=511, type="f32", state=1, tail=0,
             pad=1),
        # a toy model's parameters: latency only
        dict(name="adamw_small", op="adamw", T=24, P=65_536, grads="f32", moments=32, copy="", clip=0),
        # a model of 16 M parameters, gradients in 32 and 16 bits, scaled by the coefficient that clipping found
        dict(name="adamw_mixed", op="adamw", T=150, P=16_000_000, grads="mixed", moments=32, copy="", clip=1),
        # the largest dense shard, moments in 8 bits and a copy of the parameters in 16
        dict(name="adamw_large_8bit", op="adamw", T=300, P=200_000_000, grads="bf16", moments=8, copy="bf16", clip=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choice(["norm_fwd", "norm_bwd", "scan_fwd", "scan_bwd", "adamw"])
    kind = rng.choice(["f32", "bf16", "bf16", "f16"])
    pad = rng.choice([0, 0, 0, rng.randint(1, 64)])
    if op == "adamw":
        moments = rng.choice([32, 8])
        return dict(op=op, T=_log_int(rng, 1, 500), P=_log_int(rng, 10_000, 180_000_000 if moments == 8 else 100_000_000),
                    grads=rng.choice(["f32", "bf16", "mixed"]), moments=moments,
                    copy=rng.choice(["", "", "bf16", "f16"]), clip=rng.randint(0, 1))
    if op in ("scan_fwd", "scan_bwd"):
        D = rng.choice([16, 32, 64, 128, 256, 1_024, _log_int(rng, 8, 4_096)])
        most = 67_000_000 // D
        L = rng.choice([0, 0, 1, _log_int(rng, 1, 65_536), _log_int(rng, 1, 65_536)])
        if L == 0:
            B, n = _log_int(rng, 1, 20_000), _log_int(rng, 1, min(most, 400_000))
            tail = rng.choice([0, min(n - 1, rng.randint(0, 500))])
        else:
            L = min(L, most)
            B = _log_int(rng, 1, min(most // L, 20_000))
            n, tail = B * L, 0
        return dict(op=op, B=B, L=L, n=n, D=D, type=kind, state=rng.randint(0, 1), tail=tail, pad=pad)
    D = rng.choice([16, 32, 64, 128, 256, _log_int(rng, 8, 8_192), _log_int(rng, 64, 2_048) * 2,
                    rng.choice([1_024, 2_048, 4_096, 8_192])])
    n = _log_int(rng, 1, min(500_000, 67_000_000 // D))
    span = rng.choice([1, n, n, _log_int(rng, 1, n)])
    post, pre = rng.choice([("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("none", "layer"), ("rms", "none")])
    return dict(op=op, n=n, D=D, stream=rng.choice([kind, kind, "f32"]), type=kind, wtype=rng.choice(["f32", kind]),
                gate=rng.choice(["none", "linear", "linear", "sigmoid"]), span=span, gtype=rng.choice(["f32", kind]),
                post=post, pre=pre, bias=rng.randint(0, 1) if "layer" in (post, pre) else 0,
                alpha=rng.choice([1.0, 1.0, 0.8, 1.7]), pad=pad)


# ------------------------------------------------------------------ inputs
def _generator(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 64 + stream) & ((1 << 62) - 1))
    return g


def _normal(seed, stream, sigma, *shape, mean=0.0):
    return torch.empty(shape, device=DEV).normal_(mean, sigma, generator=_generator(seed, stream))


def _matrix(seed, stream, sigma, n, D, kind, pad, mean=0.0):
    """[n, D] values, D of every D + pad columns of a wider tensor."""
    x = torch.empty((n, D + pad), device=DEV, dtype=TYPES[kind])
    return x.normal_(mean, sigma, generator=_generator(seed, stream))[:, :D]


def _statistics(x, kind):
    mean = x.mean(1) if kind == "layer" else torch.zeros(x.shape[0], device=DEV, dtype=x.dtype)
    return mean, ((x - mean[:, None]).square().mean(1) + EPS).rsqrt()


def _sizes(case):
    """The T sizes of a model of P parameters: a few large matrices, many vectors, odd ones among them."""
    T, P = case["T"], case["P"]
    rng = random.Random(T * 1_000_003 + P)
    weight = [math.exp(rng.uniform(0.0, 7.0)) for _ in range(T)]
    spare = P - T
    sizes = [1 + int(spare * w / sum(weight)) for w in weight]
    sizes[-1] += P - sum(sizes)
    return sizes


def _kinds(case):
    """The types of the gradients: of a mixed list the short ones' are in 32 bits."""
    small = max(case["P"] // case["T"] // 8, 2)
    return [case["grads"] if case["grads"] != "mixed" else "f32" if s < small else "bf16" for s in _sizes(case)]


def _rooms(case):
    """Each tensor's room in the flat buffers of parameters and moments: whole blocks."""
    return [-(-s // BLOCK) * BLOCK for s in _sizes(case)]


def _inputs(case, seed):
    op, x = case["op"], {}
    if op == "adamw":
        sizes, rooms = _sizes(case), _rooms(case)
        total = sum(rooms)
        # (between the tensors zeros, which a step leaves zeros)
        inside = torch.zeros(total, dtype=torch.bool, device=DEV)
        for s, part in zip(sizes, inside.split(rooms)):
            part[:s] = True
        scale = torch.exp(_normal(seed, 12, 1.0, total // BLOCK)).repeat_interleave(BLOCK)
        x["param"] = _normal(seed, 1, 0.02, total) * inside
        flat = _normal(seed, 2, SIGMA, total) * scale
        x["grads"] = [p[:s].to(TYPES[k], copy=True) for p, s, k in zip(flat.split(rooms), sizes, _kinds(case))]
        m = _normal(seed, 3, SIGMA / 4, total) * scale * inside
        v = (_normal(seed, 4, SIGMA, total) * scale).square() * inside
        del flat, scale, inside
        if case["moments"] == 8:
            half = torch.full_like(m, 0.5)
            x["m"], x["m_exp"] = _encode(m, 3, half)
            x["v"], x["v_exp"] = _encode(v.sqrt(), 4, half)
        else:
            x["m"], x["v"] = m, v
        x["coef"] = torch.full((1,), 0.37, device=DEV) if case["clip"] else None
        x["copy"] = torch.zeros(total, device=DEV, dtype=TYPES[case["copy"]]) if case["copy"] else None
        x["t"] = 1_000 + int(seed) % 97
        return x
    n, D, kind, pad = case["n"], case["D"], case["type"], case["pad"]
    if op in ("scan_fwd", "scan_bwd"):
        B = case["B"]
        x["x"] = _matrix(seed, 5, 1.0, n, D, kind, pad)
        x["a"] = _matrix(seed, 6, 1.5, n, D, kind, pad, mean=2.0)
        x["h0"] = _normal(seed, 7, 0.5, B, D) if case["state"] else None
        if case["L"] == 0:
            used = n - case["tail"]
            cuts = torch.randint(0, used + 1, (B - 1,), device=DEV, generator=_generator(seed, 8))
            ends = torch.tensor([0, used], device=DEV)
            x["offsets"] = torch.cat([ends[:1], cuts.sort()[0], ends[1:]])
        else:
            x["offsets"] = None
        if op == "scan_bwd":
            x["dh"] = _matrix(seed, 9, SIGMA, n, D, kind, pad)
            x["h"] = _matrix(seed, 10, 0.4, n, D, kind, pad)
            x["dlast"] = _normal(seed, 11, SIGMA, B, D) if case["state"] else None
        return x
    stream = case["stream"]
    x["z"] = _matrix(seed, 14, 1.5, n, D, kind, pad, mean=0.1)
    G = -(-n // case["span"])
    x["gate"] = (_matrix(seed, 15, 0.5, G, D, case["gtype"], pad, mean=0.3) if case["gate"] != "none" else None)
    for at, name in ((16, "post"), (18, "pre")):
        on = case[name] != "none"
        x[name + "_weight"] = (1.0 + _normal(seed, at, 0.1, D)).to(TYPES[case["wtype"]]) if on else None
        bias = on and case["bias"] and case[name] == "layer"
        x[name + "_bias"] = _normal(seed, at + 1, 0.1, D).to(TYPES[case["wtype"]]) if bias else None
    if op == "norm_fwd":
        x["x"] = _matrix(seed, 13, 2.0, n, D, stream, pad)
        return x
    x["h"] = _matrix(seed, 20, 2.0, n, D, stream, pad)
    x["dy"] = _matrix(seed, 21, SIGMA, n, D, kind, pad) if case["pre"] != "none" else None
    x["dh"] = _matrix(seed, 22, SIGMA, n, D, stream, pad)
    for name, of in (("post", "z"), ("pre", "h")):
        mean, rstd = _statistics(x[of].float(), case[name]) if case[name] != "none" else (None, None)
        x[name + "_mean"], x[name + "_rstd"] = mean if case[name] == "layer" else None, rstd
    return x


def prepare(case, seed):
    st = dict(case=case, **_inputs(case, seed))
    if own:
        _buffers(case, st)
    return st


def _buffers(case, st):
    """Outputs, scratch and the list of tensors, which a program keeps from step to step."""
    import paper_2205_11048_amd as gba
    op = case["op"]

    def new(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=DEV)

    st["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if op == "adamw":
        sizes, rooms = _sizes(case), _rooms(case)

        def parts(name):
            return [p[:s] for p, s in zip(st[name].split(rooms), sizes)]

        exps = [r // BLOCK for r in rooms]
        kw = dict(m_exps=list(st["m_exp"].split(exps)), v_exps=list(st["v_exp"].split(exps))) if case["moments"] == 8 else {}
        st["list"] = gba.gba_adamw_list(parts("param"), st["grads"], parts("m"), parts("v"),
                                        copies=parts("copy") if case["copy"] else None, **kw)
        if case["moments"] == 8:
            st["m_values"], st["v_values"] = new(sum(rooms)), new(sum(rooms))
        return
    n, D, kind = case["n"], case["D"], TYPES[case["type"]]
    if op in ("scan_fwd", "scan_bwd"):
        st["workspace"] = new(gba.gba_recurrence_workspace_size(n, case["B"], D), dtype=torch.uint8)
        # (rows behind the last sequence are not written: they compare as zeros)
        names = ("out",) if op == "scan_fwd" else ("dx", "da")
        for name in names:
            st[name] = new(n, D, dtype=kind).zero_()
        st["last" if op == "scan_fwd" else "dh0"] = new(case["B"], D) if case["state"] else None
        return
    stream = TYPES[case["stream"]]
    if op == "norm_fwd":
        st["h"] = new(n, D, dtype=stream)
        st["y"] = new(n, D, dtype=kind) if case["pre"] != "none" else None
        for name in ("post", "pre"):
            st[name + "_mean"] = new(n) if case[name] == "layer" else None
            st[name + "_rstd"] = new(n) if case[name] != "none" else None
        return
    st["dx"], st["dz"] = new(n, D, dtype=stream), new(n, D, dtype=kind)
    st["dgate"] = new(*st["gate"].shape, dtype=st["gate"].dtype) if st["gate"] is not None else None
    for name in ("post_weight", "post_bias", "pre_weight", "pre_bias"):
        st["d" + name] = new(D) if st[name] is not None else None
    st["workspace"] = new(gba.gba_residual_norm_grad_workspace_size(n, D), dtype=torch.uint8)


# ------------------------------------------------------------------ the calls
def _run_own(st):
    import paper_2205_11048_amd as gba
    case = st["case"]
    op = case["op"]
    if op == "adamw":
        st["t"] += 1
        gba.gba_adamw(st["list"], LR, BETA1, BETA2, ADAM_EPS, DECAY, st["t"], seed=SEED, coef=st["coef"],
                      err=st["err"])
        if case["moments"] == 32:
            return _adamw_out(st)
        gba.gba_moments_read(st["m"], st["m_exp"], gba.MOMENT_M, st["m_values"])
        gba.gba_moments_read(st["v"], st["v_exp"], gba.MOMENT_V, st["v_values"])
        return {"param": st["param"], "m": st["m_values"], "v": st["v_values"], "copy": st["copy"]}
    if op == "scan_fwd":
        gba.gba_recurrence(st["x"], st["a"], st["out"], offsets=st["offsets"], length=case["L"], h0=st["h0"],
                           h_last=st["last"], workspace=st["workspace"], err=st["err"])
        return {"h": st["out"], "last": st["last"]}
    if op == "scan_bwd":
        gba.gba_recurrence_grad(st["dh"], st["x"], st["a"], st["h"], st["dx"], st["da"], offsets=st["offsets"],
                                length=case["L"], h0=st["h0"], dh_last=st["dlast"], dh0=st["dh0"],
                                workspace=st["workspace"], err=st["err"])
        return {"dx": st["dx"], "da": st["da"], "dh0": st["dh0"]}
    norms = dict(gate=st["gate"], gate_kind=_gate_kind(gba, case), gate_span=case["span"], alpha=case["alpha"],
                 eps=EPS, post=_norm_kind(gba, case["post"]), pre=_norm_kind(gba, case["pre"]),
                 post_weight=st["post_weight"], pre_weight=st["pre_weight"], post_mean=st["post_mean"],
                 post_rstd=st["post_rstd"], pre_mean=st["pre_mean"], pre_rstd=st["pre_rstd"])
    if op == "norm_fwd":
        gba.gba_residual_norm(st["x"], st["z"], st["h"], st["y"], post_bias=st["post_bias"], pre_bias=st["pre_bias"],
                              **norms)
        return {k: st[k] for k in ("h", "y", "post_mean", "post_rstd", "pre_mean", "pre_rstd")}
    gba.gba_residual_norm_grad(st["dy"], st["dh"], st["z"], st["h"], st["dx"], st["dz"], st["workspace"],
                               post_bias=st["post_bias"], dgate=st["dgate"], dpost_weight=st["dpost_weight"],
                               dpost_bias=st["dpost_bias"], dpre_weight=st["dpre_weight"],
                               dpre_bias=st["dpre_bias"], **norms)
    return {k: st[k] for k in ("dx", "dz", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")}


def _norm_kind(gba, name):
    return {"none": gba.ROW_NORM_NONE, "layer": gba.ROW_NORM_LAYER, "rms": gba.ROW_NORM_RMS}[name]


def _gate_kind(gba, case):
    return {"none": gba.GATE_NONE, "linear": gba.GATE_LINEAR, "sigmoid": gba.GATE_SIGMOID}[case["gate"]]


def run(st):
    if own:
        return _run_own(st)
    op = st["case"]["op"]
    if op == "adamw":
        return _adamw(st)
    if op == "scan_fwd":
        return _scan(st)
    if op == "scan_bwd":
        return _scan_grad(st)
    return _norm(st) if op == "norm_fwd" else _norm_grad(st)


# ---- norms, gate and residual
def _normed(x, kind, weight, bias, mean=None, rstd=None):
    """(x normalised, the result, the statistics)"""
    if kind == "none":
        return None, x, None, None
    if rstd is None:
        mean, rstd = _statistics(x, kind)
    xh = (x - mean[:, None] if kind == "layer" else x) * rstd[:, None]
    y = xh * weight.float()
    return xh, (y if bias is None else y + bias.float()), (mean if kind == "layer" else None), rstd


def _gate_rows(case, gate, n):
    """A factor for every row, [n, D] or [1, D]."""
    g = gate.float()
    if case["gate"] == "sigmoid":
        g = torch.sigmoid(g)
    return g if g.shape[0] in (1, n) else g.repeat_interleave(case["span"], 0)[:n]


def _norm(st):
    case = st["case"]
    _, u, mean_z, rstd_z = _normed(st["z"].float(), case["post"], st["post_weight"], st["post_bias"])
    if st["gate"] is not None:
        u = u * _gate_rows(case, st["gate"], case["n"])
    h = (st["x"].float() * case["alpha"] + u).to(TYPES[case["stream"]])
    _, y, mean_h, rstd_h = _normed(h.float(), case["pre"], st["pre_weight"], st["pre_bias"])
    y = y.to(TYPES[case["type"]]) if case["pre"] != "none" else None
    return {"h": h, "y": y, "post_mean": mean_z, "post_rstd": rstd_z, "pre_mean": mean_h, "pre_rstd": rstd_h}


def _normed_grad(d, xh, rstd, kind, weight):
    """The gradient of what was normalised."""
    h = d * weight.float()
    along = (h * xh).mean(1, keepdim=True)
    if kind == "layer":
        h = h - h.mean(1, keepdim=True)
    return (h - xh * along) * rstd[:, None]


def _norm_grad(st):
    case, n = st["case"], st["case"]["n"]
    d, out = st["dh"].float(), {}
    if case["pre"] != "none":
        dy = st["dy"].float()
        xh = _normed(st["h"].float(), case["pre"], st["pre_weight"], None, st["pre_mean"], st["pre_rstd"])[0]
        out["dpre_weight"] = (dy * xh).sum(0)
        out["dpre_bias"] = dy.sum(0) if st["pre_bias"] is not None else None
        d = d + _normed_grad(dy, xh, st["pre_rstd"], case["pre"], st["pre_weight"])
    out["dx"] = (d * case["alpha"]).to(TYPES[case["stream"]])
    zh, u, _, _ = _normed(st["z"].float(), case["post"], st["post_weight"], st["post_bias"], st["post_mean"],
                          st["post_rstd"])
    if st["gate"] is not None:
        g = _gate_rows(case, st["gate"], n)
        dg = d * u
        d = d * g
        span = min(case["span"], n)
        if span > 1:
            G = st["gate"].shape[0]
            rows = torch.zeros((G * span, case["D"]), device=DEV)
            rows[:n] = dg
            dg = rows.reshape(G, span, -1).sum(1)
        if case["gate"] == "sigmoid":
            s = torch.sigmoid(st["gate"].float())
            dg = dg * s * (1.0 - s)
        out["dgate"] = dg.to(TYPES[case["gtype"]])
    if case["post"] != "none":
        out["dpost_weight"] = (d * zh).sum(0)
        out["dpost_bias"] = d.sum(0) if st["post_bias"] is not None else None
        d = _normed_grad(d, zh, st["post_rstd"], case["post"], st["post_weight"])
    out["dz"] = d.to(TYPES[case["type"]])
    return out


# ---- the recurrence
def _places(case, offsets):
    """(sequences that are not empty, their first and last positions; rows in sequences)"""
    if offsets is None:
        first = torch.arange(case["B"], device=DEV) * case["L"]
        return torch.arange(case["B"], device=DEV), first, first + case["L"] - 1, case["n"]
    keep = (offsets[1:] > offsets[:-1]).nonzero()[:, 0]
    return keep, offsets[keep], offsets[keep + 1] - 1, case["n"] - case["tail"]


def _affine_scan(F, S, steps):
    """S[t] + F[t] * (S[t-1] + F[t-1] * ...) along the first axis, by doubling; in place."""
    k = 1
    while k < steps:
        S[k:] += F[k:] * S[:-k]
        F[k:] = F[k:] * F[:-k]
        k *= 2
    return S


def _steps(case):
    return case["L"] or case["n"]


def _scan(st):
    case = st["case"]
    keep, first, last, rows = _places(case, st["offsets"])
    x, a = st["x"][:rows].float(), st["a"][:rows].float()
    F, S = torch.sigmoid(a), torch.sigmoid(-a) * x
    if st["h0"] is not None:
        S[first] += F[first] * st["h0"][keep]
    F[first] = 0.0
    S = _affine_scan(F, S, _steps(case))
    h = torch.zeros((case["n"], case["D"]), device=DEV, dtype=TYPES[case["type"]])
    h[:rows] = S.to(h.dtype)
    if st["h0"] is None:
        return {"h": h, "last": None}
    state = st["h0"].clone()
    state[keep] = S[last]
    return {"h": h, "last": state}


def _scan_grad(st):
    case = st["case"]
    keep, first, last, rows = _places(case, st["offsets"])
    x, a, d = st["x"][:rows].float(), st["a"][:rows].float(), st["dh"][:rows].float()
    f, i = torch.sigmoid(a), torch.sigmoid(-a)
    # g[t] = d[t] + f[t + 1] g[t + 1], from the end
    F = torch.zeros_like(f)
    F[:-1] = f[1:]
    F[last] = 0.0
    d = d.flip(0)
    if st["dlast"] is not None:
        d[rows - 1 - last] += st["dlast"][keep]
    g = _affine_scan(F.flip(0), d, _steps(case)).flip(0)
    before = torch.zeros_like(x)
    before[1:] = st["h"][:rows - 1].float()
    before[first] = st["h0"][keep] if st["h0"] is not None else 0.0
    out = {}
    for name, v in (("dx", g * i), ("da", g * (before - x) * f * i)):
        out[name] = torch.zeros((case["n"], case["D"]), device=DEV, dtype=TYPES[case["type"]])
        out[name][:rows] = v.to(out[name].dtype)
    out["dh0"] = None
    if st["h0"] is not None:
        out["dh0"] = st["dlast"].clone()
        out["dh0"][keep] = f[first] * g[first]
    return out


# ---- AdamW
def _mix(x):
    """32 bits mixed, in int64."""
    low = 0xFFFFFFFF
    x = x ^ (x >> 16)
    x = (x * 0xB7E15163) & low
    x = x ^ (x >> 15)
    x = (x * 0x9E3779B1) & low
    return x ^ (x >> 16)


def _uniforms(case, t):
    """Two numbers in (0, 1) for every place of the flat buffers, multiples of 2^-17: of the seed, the step, the
    tensor, and the block and the place in it."""
    blocks = torch.tensor([r // BLOCK for r in _rooms(case)], device=DEV)
    tensor = torch.arange(case["T"], device=DEV).repeat_interleave(blocks)
    block = torch.arange(tensor.numel(), device=DEV) - (blocks.cumsum(0) - blocks)[tensor]
    low = 0xFFFFFFFF
    key = _mix((_mix(torch.full_like(tensor, (SEED + t) & low)) + tensor) & low)
    key = _mix((key + block) & low)
    bits = _mix((key[:, None] + torch.arange(BLOCK, device=DEV)) & low).reshape(-1)
    return ((bits & 0xFFFF).float() + 0.5) * 2.0 ** -16, ((bits >> 16).float() + 0.5) * 2.0 ** -16


def _encode(x, mantissa, u):
    """Values of blocks of 256 as a code of 4 exponent and ``mantissa`` mantissa bits (and a sign where there are 3
    of them), with an exponent for each block: the smallest power of two that brings the block's largest value to
    no more than the largest code, 2 - 2^-mantissa.  What lies between two codes is rounded up where its fraction
    and u are 1 or more together."""
    y = x.reshape(-1, BLOCK).double()
    top = y.abs().amax(1)
    exp = torch.ceil(torch.log2(top / (2.0 - 2.0 ** -mantissa)).clamp(-200, 200))
    for _ in range(2):   # (a logarithm may be off next to a power of two)
        exp = torch.where(top > (2.0 - 2.0 ** -mantissa) * torch.exp2(exp), exp + 1, exp)
        exp = torch.where(top <= (2.0 - 2.0 ** -mantissa) * torch.exp2(exp - 1), exp - 1, exp)
    exp = exp.clamp(-126, 127)
    y *= torch.exp2(-exp)[:, None]
    sign = y < 0
    y = y.abs()
    e = torch.where(y > 0, torch.frexp(y)[1].clamp(min=-13) - 1, -14)     # y < 2^(e + 1)
    places = 23 - mantissa
    f = torch.round(torch.ldexp(y, mantissa + places - e)) * 2.0 ** -places    # (the fraction in as many bits)
    f = torch.floor(f + u.reshape(f.shape))
    code = (f + (e + 14) * 2 ** mantissa).clamp(max=2 ** (4 + mantissa) - 1)   # (without the leading bit, which carries)
    if mantissa == 3:
        code += 128 * sign
    return code.to(torch.uint8).reshape(-1), torch.where(top > 0, exp + 127, 0).to(torch.uint8)


def _decode(code, exp, mantissa):
    c = code.reshape(-1, BLOCK).int()
    sign = 1 - 2 * (c >> 7) if mantissa == 3 else 1
    c = c & (2 ** (4 + mantissa) - 1)
    e = (c >> mantissa).clamp(min=1)
    f = c - ((e - 1) << mantissa)
    v = sign * f * torch.exp2((e - 15 - mantissa).double()) * torch.exp2(exp.double() - 127)[:, None]
    return v.float().reshape(-1)


def _flat_grads(st):
    case = st["case"]
    gaps = [torch.zeros(r - s, device=DEV) for r, s in zip(_rooms(case), _sizes(case))]
    return torch.cat([p for g, gap in zip(st["grads"], gaps) for p in (g.float(), gap)])


def _adamw(st):
    case = st["case"]
    st["t"] += 1
    t = st["t"]
    g = _flat_grads(st)
    if case["clip"]:
        g *= st["coef"]
    eight = case["moments"] == 8
    m = _decode(st["m"], st["m_exp"], 3) if eight else st["m"]
    v = _decode(st["v"], st["v_exp"], 4).square() if eight else st["v"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    root = v.sqrt()
    step = (m / (1.0 - BETA1 ** t)) / (root / math.sqrt(1.0 - BETA2 ** t) + ADAM_EPS)
    st["param"].mul_(1.0 - LR * DECAY).sub_(step * LR)
    if case["copy"]:
        st["copy"].copy_(st["param"])
    if eight:
        um, uv = _uniforms(case, t)
        codes = (*_encode(m, 3, um), *_encode(root, 4, uv))
        for name, value in zip(("m", "m_exp", "v", "v_exp"), codes):
            st[name].copy_(value)
    else:
        st["m"].copy_(m)
        st["v"].copy_(v)
    return _adamw_out(st)


def _adamw_out(st):
    """The updated buffers; of moments in 8 bits the values that they stand for (m, and the root of v)."""
    if st["case"]["moments"] == 8:
        m, v = _decode(st["m"], st["m_exp"], 3), _decode(st["v"], st["v_exp"], 4)
    else:
        m, v = st["m"], st["v"]
    return {"param": st["param"], "m": m, "v": v, "copy": st["copy"]}


# ------------------------------------------------------------------ accounts
def work(case):
    """Inputs read once, outputs written once."""
    op = case["op"]
    if op == "adamw":
        P = case["P"]
        grads = sum(s * SIZE[k] for s, k in zip(_sizes(case), _kinds(case)))
        moments = 16 * P if case["moments"] == 32 else 4 * P + 4 * P / BLOCK
        return {"bytes": float(8 * P + grads + moments + (SIZE[case["copy"]] * P if case["copy"] else 0)),
                "flops": 16.0 * P}
    n, D, b = case["n"], case["D"], SIZE[case["type"]]
    if op in ("scan_fwd", "scan_bwd"):
        rows = n - case["tail"]
        small = 8 * (case["B"] + 1) * (case["L"] == 0)
        states = case["state"] * case["B"] * D * 4
        if op == "scan_fwd":
            return {"bytes": 3.0 * rows * D * b + small + 2 * states, "flops": 6.0 * rows * D}
        return {"bytes": 6.0 * rows * D * b + small + 3 * states, "flops": 12.0 * rows * D}
    s = SIZE[case["stream"]]
    G = -(-n // case["span"]) if case["gate"] != "none" else 0
    norms = (case["post"] != "none") + (case["pre"] != "none")
    stats = 4 * n * sum({"none": 0, "rms": 1, "layer": 2}[case[k]] for k in ("post", "pre"))
    pre = case["pre"] != "none"
    params = D * (norms + case["bias"] * sum(case[k] == "layer" for k in ("post", "pre")))
    gate = G * D * SIZE[case["gtype"]]
    if op == "norm_fwd":
        return {"bytes": float(n * D * (2 * s + b * (1 + pre)) + stats + gate + params * SIZE[case["wtype"]]),
                "flops": 16.0 * n * D}
    return {"bytes": float(n * D * ((2 + pre) * s + b * (2 + pre)) + stats + 2 * gate + params * (4 + SIZE[case["wtype"]])),
            "flops": 30.0 * n * D}


# ------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """What ``run`` returns, from the definitions in float64; None in the place of what is held in 8 bits."""
    x = _inputs(case, seed)
    return {"adamw": _exact_adamw, "scan_fwd": _exact_scan, "scan_bwd": _exact_scan_grad, "norm_fwd": _exact_norm,
            "norm_bwd": _exact_norm_grad}[case["op"]](case, x)


def _exact_adamw(case, x):
    eight, t = case["moments"] == 8, x["t"] + 1
    coef = x["coef"].double() if case["clip"] else 1.0
    at, out = 0, {"param": x["param"].double(), "m": None, "v": None, "copy": None}
    if not eight:
        out["m"], out["v"] = x["m"].double(), x["v"].double()
    for s, room, g in zip(_sizes(case), _rooms(case), x["grads"]):
        here, blocks = slice(at, at + room), slice(at // BLOCK, (at + room) // BLOCK)
        g = g.double() * coef
        if eight:
            m = _decode(x["m"][here], x["m_exp"][blocks], 3)[:s].double()
            v = _decode(x["v"][here], x["v_exp"][blocks], 4)[:s].double().square()
        else:
            m, v = out["m"][here][:s], out["v"][here][:s]
        m = BETA1 * m + (1.0 - BETA1) * g
        v = BETA2 * v + (1.0 - BETA2) * g * g
        p = out["param"][here][:s]
        p -= LR * (m / (1.0 - BETA1 ** t) / ((v / (1.0 - BETA2 ** t)).sqrt() + ADAM_EPS) + DECAY * p)
        if not eight:
            out["m"][here][:s], out["v"][here][:s] = m, v
        at += room
    if case["copy"]:
        out["copy"] = out["param"]
    return out


def _lengths(case, x):
    """(starts, lengths, in the order of falling length; how many sequences have more than t positions)"""
    if x["offsets"] is None:
        starts = torch.arange(case["B"], device=DEV) * case["L"]
        lengths = torch.full((case["B"],), case["L"], device=DEV)
    else:
        starts, lengths = x["offsets"][:-1], x["offsets"][1:] - x["offsets"][:-1]
    order = torch.argsort(lengths, descending=True, stable=True)
    longest = int(lengths.max())
    count = torch.bincount(lengths, minlength=longest + 1).flip(0).cumsum(0).flip(0)[1:].tolist()
    return order, starts[order], lengths[order], count


def _exact_scan(case, x):
    order, starts, lengths, count = _lengths(case, x)
    if len(count) > 140_000:
        return None
    f = 1.0 / (1.0 + torch.exp(-x["a"].double()))
    v = (1.0 - f) * x["x"].double()
    h = torch.zeros_like(f)
    state = torch.zeros((case["B"], case["D"]), dtype=torch.float64, device=DEV)
    if x["h0"] is not None:
        state += x["h0"][order]
    for t, k in enumerate(count):
        at = starts[:k] + t
        state[:k] = f[at] * state[:k] + v[at]
        h[at] = state[:k]
    last = torch.empty_like(state)
    last[order] = state
    return {"h": h, "last": last if x["h0"] is not None else None}


def _exact_scan_grad(case, x):
    order, starts, lengths, count = _lengths(case, x)
    if len(count) > 140_000:
        return None
    a = x["a"].double()
    f, i = 1.0 / (1.0 + torch.exp(-a)), 1.0 / (1.0 + torch.exp(a))
    g = torch.zeros_like(f)
    d = x["dh"].double()
    zero = torch.zeros((case["B"], case["D"]), dtype=torch.float64, device=DEV)
    carry = x["dlast"][order].double() if x["dlast"] is not None else zero.clone()
    h0 = x["h0"][order].double() if x["h0"] is not None else zero
    before = torch.zeros_like(f)
    before[1:] = x["h"][:-1].double()
    before[starts[:count[0] if count else 0]] = h0[:count[0] if count else 0]
    for t in range(len(count) - 1, -1, -1):
        k = count[t]
        at = starts[:k] + t
        now = d[at] + carry[:k]
        g[at] = now
        carry[:k] = f[at] * now
    dh0 = torch.empty_like(carry)
    dh0[order] = carry
    return {"dx": g * i, "da": g * (before - x["x"].double()) * f * i, "dh0": dh0 if x["h0"] is not None else None}


def _exact_rows(x, kind):
    mean = x.sum(1, keepdim=True) / x.shape[1] if kind == "layer" else 0.0
    d = x - mean
    rstd = 1.0 / torch.sqrt((d * d).sum(1, keepdim=True) / x.shape[1] + EPS)
    return mean, rstd


def _exact_gate(case, x):
    g = x["gate"].double()
    g = 1.0 / (1.0 + torch.exp(-g)) if case["gate"] == "sigmoid" else g
    return g[torch.arange(case["n"], device=DEV) // case["span"]]


def _exact_norm(case, x):
    out = {}
    u = x["z"].double()
    if case["post"] != "none":
        mean, rstd = _exact_rows(u, case["post"])
        u = (u - mean) * rstd * x["post_weight"].double()
        if x["post_bias"] is not None:
            u += x["post_bias"].double()
        out["post_mean"], out["post_rstd"] = mean[:, 0] if case["post"] == "layer" else None, rstd[:, 0]
    if x["gate"] is not None:
        u *= _exact_gate(case, x)
    out["h"] = u + case["alpha"] * x["x"].double()
    if case["pre"] != "none":
        h = out["h"].to(TYPES[case["stream"]]).double()     # what is normalised is the stream as it is held
        mean, rstd = _exact_rows(h, case["pre"])
        y = (h - mean) * rstd * x["pre_weight"].double()
        out["y"] = y + x["pre_bias"].double() if x["pre_bias"] is not None else y
        out["pre_mean"], out["pre_rstd"] = mean[:, 0] if case["pre"] == "layer" else None, rstd[:, 0]
    return out


def _exact_back(d, xh, rstd, weight, kind):
    h = d * weight.double()
    D = d.shape[1]
    mean = h.sum(1, keepdim=True) / D if kind == "layer" else 0.0
    return rstd * (h - mean - xh * ((h * xh).sum(1, keepdim=True) / D))


def _exact_norm_grad(case, x):
    out, d = {}, x["dh"].double()

    def hat(of, name):
        mean = x[name + "_mean"].double()[:, None] if case[name] == "layer" else 0.0
        rstd = x[name + "_rstd"].double()[:, None]
        return (x[of].double() - mean) * rstd, rstd

    if case["pre"] != "none":
        xh, rstd = hat("h", "pre")
        dy = x["dy"].double()
        out["dpre_weight"] = (dy * xh).sum(0)
        if x["pre_bias"] is not None:
            out["dpre_bias"] = dy.sum(0)
        d = d + _exact_back(dy, xh, rstd, x["pre_weight"], case["pre"])
    out["dx"] = case["alpha"] * d
    u = x["z"].double()
    if case["post"] != "none":
        zh, rstd = hat("z", "post")
        u = zh * x["post_weight"].double()
        if x["post_bias"] is not None:
            u += x["post_bias"].double()
    if x["gate"] is not None:
        s = _exact_gate(case, x)
        each = d * u
        if case["gate"] == "sigmoid":
            each *= s * (1.0 - s)
        at = torch.arange(case["n"], device=DEV) // case["span"]
        out["dgate"] = torch.zeros(x["gate"].shape, dtype=torch.float64, device=DEV).index_add_(0, at, each)
        d = d * s
    if case["post"] != "none":
        out["dpost_weight"] = (d * zh).sum(0)
        if x["post_bias"] is not None:
            out["dpost_bias"] = d.sum(0)
        d = _exact_back(d, zh, rstd, x["post_weight"], case["post"])
    out["dz"] = d
    return out
