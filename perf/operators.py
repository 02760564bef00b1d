"""Performance cases of the residual block's operators: the norm over a model's columns, the linear projection with bias,
activation and residual, and the gated projection pair of the feed-forward half, each forward and backward.

A case is a dict of plain values: ``op`` and ``direction``, the sizes (M tokens, K input columns, N output columns; the
norm has D columns), the type of the activations and weights, and which of the optional parts are there.  Norm weights,
biases, row statistics and the gradients of weights that are vectors are single precision throughout; a backward case is
given what the forward call left (row statistics, pre-activations), as a training program has it in hand.

4096 columns are those of the 8 heads of 512 that the cell's configurations use, 16384 tokens those of the training
configuration (2 sequences of 8192); 10944 is 8/3 of 4096, rounded up to whole blocks of 64.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6


def _norm(name, direction, M, D, kind="rms", dtype="bf16", residual=False):
    return {"name": name, "op": "norm", "direction": direction, "M": M, "D": D, "kind": kind, "dtype": dtype,
            "residual": residual}


def _linear(name, direction, M, K, N, act="none", dtype="bf16", bias=True, residual=False, keep=False):
    return {"name": name, "op": "linear", "direction": direction, "M": M, "K": K, "N": N, "act": act, "dtype": dtype,
            "bias": bias, "residual": residual, "keep": keep}


def _gated(name, direction, M, K, N, act="silu", dtype="bf16", bias=False, keep=False):
    return {"name": name, "op": "gated", "direction": direction, "M": M, "K": K, "N": N, "act": act, "dtype": dtype,
            "bias": bias, "keep": keep}


def listed():
    return [
        # one token's pre-norm while generating: the smallest call of all, two per block and token
        _norm("norm_one_token", "fwd", 1, 4096),
        # the pre-norm of the training configuration, forward
        _norm("norm_prompt", "fwd", 16384, 4096),
        # the same backward with LayerNorm; the gradient that goes round the norm is added on the way
        _norm("norm_train", "bwd", 16384, 4096, kind="layer", residual=True),
        # single precision, a width that no vector load divides
        _norm("norm_ragged_f32", "bwd", 2999, 1365, kind="layer", dtype="f32"),
        # one token through the projection out of the heads
        _linear("linear_one_token", "fwd", 1, 4096, 4096, residual=True),
        # a prompt of ordinary, odd length through it
        _linear("linear_prompt", "fwd", 2000, 4096, 4096, residual=True),
        # training a projection of that width on one long sequence
        _linear("linear_train", "bwd", 8192, 4096, 4096),
        # single precision with an activation, nothing of which is a multiple of a tile
        _linear("linear_ragged_f32", "fwd", 333, 1000, 777, act="gelu", dtype="f32", keep=True),
        # four sequences generating together through the wide half of the feed-forward block: weights read once
        _gated("gated_decode", "fwd", 4, 4096, 10944),
        # a long sequence through it, with what the backward pass needs kept
        _gated("gated_train_fwd", "fwd", 8192, 4096, 10944, keep=True),
        # and its backward pass: the largest call
        _gated("gated_train_bwd", "bwd", 8192, 4096, 10944),
        # a small odd one: output columns whose rows start at odd addresses, biases, the other activation
        _gated("gated_ragged", "bwd", 1000, 1000, 1365, act="gelu", bias=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _columns(rng, lo, hi):
    """A width: a multiple of 64 in half of the draws, of 8 in a quarter, anything in the rest."""
    x, step = _log_int(rng, lo, hi), rng.choice([64, 64, 8, 1])
    return max(step, x // step * step)


def _cost(c):
    """A rough time of one pass in seconds (not a floor): keeps drawn cases below the largest listed one."""
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / (1e14 if c["dtype"] == "f32" else 1e15)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op, direction = rng.choice(["norm", "linear", "gated"]), rng.choice(["fwd", "bwd"])
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        if op == "norm":
            c = _norm("", direction, _log_int(rng, 1, 32768), _columns(rng, 64, 8192), rng.choice(["rms", "layer"]), dtype,
                      direction == "bwd" and rng.random() < 0.5)
        elif op == "linear":
            c = _linear("", direction, _log_int(rng, 1, 16384), _columns(rng, 64, 8192), _columns(rng, 64, 8192),
                        rng.choice(["none", "none", "silu", "gelu", "relu"]), dtype, rng.random() < 0.5,
                        direction == "fwd" and rng.random() < 0.5, direction == "fwd" and rng.random() < 0.3)
        else:
            c = _gated("", direction, _log_int(rng, 1, 8192), _columns(rng, 64, 4096), _columns(rng, 64, 10944),
                       rng.choice(["silu", "silu", "gelu", "relu"]), dtype, rng.random() < 0.3,
                       direction == "fwd" and rng.random() < 0.5)
        del c["name"]
        if _cost(c) <= most:
            return c


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    c, t, gen = case, _type(case), torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=t):
        return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)

    s = {"case": dict(c), "out": {}}
    M = c["M"]
    if c["op"] == "norm":
        D = c["D"]
        # the residual stream: columns of different size, rows that have drifted from zero
        scale = torch.exp(0.5 * torch.randn(D, generator=gen, device="cuda"))
        x = torch.randn((M, D), generator=gen, device="cuda") * scale
        s["x"] = (x + 0.3 * torch.randn((M, 1), generator=gen, device="cuda")).to(t)
        s["gamma"] = normal(D, std=0.2, mean=1.0, dtype=torch.float32)
        s["beta"] = normal(D, std=0.2, dtype=torch.float32) if c["kind"] == "layer" else None
        if c["direction"] == "bwd":
            s["dy"] = normal(M, D)
            s["d_residual"] = normal(M, D) if c["residual"] else None
            xd = s["x"].double()
            mean = xd.mean(-1) if c["kind"] == "layer" else torch.zeros(M, dtype=torch.float64, device="cuda")
            s["rstd"] = (((xd - mean[:, None]) ** 2).mean(-1) + EPS).rsqrt().float()
            s["mean"] = mean.float() if c["kind"] == "layer" else None
        return s
    K, N = c["K"], c["N"]
    s["x"] = normal(M, K)
    if c["op"] == "linear":
        s["w"] = normal(N, K, std=K ** -0.5)
        s["bias"] = normal(N, std=0.1, dtype=torch.float32) if c["bias"] else None
        if c["direction"] == "fwd":
            s["residual"] = normal(M, N) if c["residual"] else None
        else:
            s["dy"] = normal(M, N)
            s["z"] = _product(s["x"], s["w"], s["bias"]).to(t) if c["act"] != "none" else None
        return s
    s["w_gate"], s["w_up"] = normal(N, K, std=K ** -0.5), normal(N, K, std=K ** -0.5)
    s["b_gate"] = normal(N, std=0.1, dtype=torch.float32) if c["bias"] else None
    s["b_up"] = normal(N, std=0.1, dtype=torch.float32) if c["bias"] else None
    if c["direction"] == "bwd":
        s["dh"] = normal(M, N)
        s["a"] = _product(s["x"], s["w_gate"], s["b_gate"]).to(t)
        s["u"] = _product(s["x"], s["w_up"], s["b_up"]).to(t)
    return s


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    return {"norm": {"fwd": _norm_fwd, "bwd": _norm_bwd}, "linear": {"fwd": _linear_fwd, "bwd": _linear_bwd},
            "gated": {"fwd": _gated_fwd, "bwd": _gated_bwd}}[c["op"]][c["direction"]](state, c)


# ---- the framework's calls ------------------------------------------------------------------------------------------
def _run_own(s, c):
    # the program owns its output tensors and workspaces: the first call leaves them in s["out"], later ones write there
    import paper_2503_14376_amd as tfla
    fwd, o = c["direction"] == "fwd", s["out"]
    if c["op"] == "norm":
        kind = tfla.NORM_LAYER if c["kind"] == "layer" else tfla.NORM_RMS
        if fwd:
            tfla.norm_fwd(s["x"], s["gamma"], s["beta"], norm_kind=kind, norm_eps=EPS, out=o)
            return {k: o[k] for k in (("y", "rstd", "mean") if c["kind"] == "layer" else ("y", "rstd"))}
        tfla.norm_bwd(s["x"], s["dy"], s["rstd"], s["mean"], s["gamma"], s["d_residual"], norm_kind=kind,
                      want_dbeta=c["kind"] == "layer", out=o)
        return {k: o[k] for k in (("dx", "dgamma", "dbeta") if c["kind"] == "layer" else ("dx", "dgamma"))}
    act = {"none": tfla.ACT_NONE, "silu": tfla.ACT_SILU, "gelu": tfla.ACT_GELU, "relu": tfla.ACT_RELU}[c["act"]]
    if c["op"] == "linear":
        if fwd:
            tfla.linear_fwd(s["x"], s["w"], s["bias"], s["residual"], act=act, keep_pre=c["keep"], out=o)
            return {k: o[k] for k in (("y", "z") if c["keep"] else ("y",))}
        tfla.linear_bwd(s["x"], s["w"], s["dy"], s["z"], act=act, want_db=c["bias"], out=o)
        return {k: o[k] for k in (("dx", "dw", "db") if c["bias"] else ("dx", "dw"))}
    if fwd:
        tfla.gated_fwd(s["x"], s["w_gate"], s["w_up"], s["b_gate"], s["b_up"], act=act, keep_pre=c["keep"], out=o)
        return {k: o[k] for k in (("h", "a", "u") if c["keep"] else ("h",))}
    tfla.gated_bwd(s["x"], s["w_gate"], s["w_up"], s["a"], s["u"], s["dh"], act=act, want_db=c["bias"], out=o)
    names = ("dx", "dw_gate", "dw_up") + (("db_gate", "db_up") if c["bias"] else ())
    return {k: o[k] for k in names}


# ---- the plain forms: single precision, rounded once at the end ---------------------------------------------------
def _product(x, w, bias):
    z = x.float() @ w.float().t()
    return z if bias is None else z + bias


def _act(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z.clamp_min(0) if act == "relu" else z


def _act_grad(z, act):
    if act == "silu":
        g = 1 / (1 + torch.exp(-z))
        return g * (1 + z * (1 - g))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return (z > 0).to(z.dtype) if act == "relu" else torch.ones_like(z)


def _norm_fwd(s, c):
    x, o = s["x"].float(), {}
    if c["kind"] == "layer":
        mean = x.sum(-1, keepdim=True) / c["D"]
        x = x - mean
        o["mean"] = mean[:, 0]
    rstd = 1 / torch.sqrt((x * x).sum(-1, keepdim=True) / c["D"] + EPS)
    y = x * rstd * s["gamma"]
    o["y"] = (y if s["beta"] is None else y + s["beta"]).to(_type(c))
    o["rstd"] = rstd[:, 0]
    return o


def _norm_bwd(s, c):
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    layer = c["kind"] == "layer"
    xh = (x - s["mean"][:, None] if layer else x) * rstd
    g = dy * s["gamma"]
    dx = g - xh * ((g * xh).sum(-1, keepdim=True) / c["D"])
    if layer:
        dx = dx - g.sum(-1, keepdim=True) / c["D"]
    dx = dx * rstd
    if s["d_residual"] is not None:
        dx = dx + s["d_residual"].float()
    o = {"dx": dx.to(_type(c)), "dgamma": (dy * xh).sum(0)}
    if layer:
        o["dbeta"] = dy.sum(0)
    return o


def _linear_fwd(s, c):
    z = _product(s["x"], s["w"], s["bias"])
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    o = {"y": y.to(_type(c))}
    if c["keep"]:
        o["z"] = z.to(_type(c))
    return o


def _linear_bwd(s, c):
    t, dz = _type(c), s["dy"].float()
    if c["act"] != "none":
        dz = dz * _act_grad(s["z"].float(), c["act"])
    o = {"dx": (dz @ s["w"].float()).to(t), "dw": (dz.t() @ s["x"].float()).to(t)}
    if c["bias"]:
        o["db"] = dz.sum(0)
    return o


def _gated_fwd(s, c):
    t = _type(c)
    a, u = _product(s["x"], s["w_gate"], s["b_gate"]), _product(s["x"], s["w_up"], s["b_up"])
    o = {"h": (_act(a, c["act"]) * u).to(t)}
    if c["keep"]:
        o["a"], o["u"] = a.to(t), u.to(t)
    return o


def _gated_bwd(s, c):
    t, x = _type(c), s["x"].float()
    a, u, dh = s["a"].float(), s["u"].float(), s["dh"].float()
    da, du = dh * u * _act_grad(a, c["act"]), dh * _act(a, c["act"])
    o = {"dx": (da @ s["w_gate"].float() + du @ s["w_up"].float()).to(t), "dw_gate": (da.t() @ x).to(t),
         "dw_up": (du.t() @ x).to(t)}
    if c["bias"]:
        o["db_gate"], o["db_up"] = da.sum(0), du.sum(0)
    return o


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    c = case
    e, M, bwd = (2 if c["dtype"] == "bf16" else 4), c["M"], c["direction"] == "bwd"
    if c["op"] == "norm":
        D, layer = c["D"], c["kind"] == "layer"
        stats, vectors = 4 * M * (2 if layer else 1), 4 * D * ((3 if layer else 2) if bwd else (2 if layer else 1))
        tensors = (3 + c["residual"]) if bwd else 2
        return {"bytes": tensors * M * D * e + stats + vectors, "flops": M * D * (14 if bwd else 7)}
    K, N = c["K"], c["N"]
    if c["op"] == "linear":
        vector = 4 * N if c["bias"] else 0
        if bwd:
            mn = 1 + (c["act"] != "none")
            return {"bytes": e * (2 * M * K + 2 * N * K + mn * M * N) + vector, "flops": 4 * M * N * K}
        return {"bytes": e * (M * K + N * K + M * N * (1 + c["residual"] + c["keep"])) + vector, "flops": 2 * M * N * K}
    vector = 8 * N if c["bias"] else 0
    if bwd:
        return {"bytes": e * (2 * M * K + 4 * N * K + 3 * M * N) + vector, "flops": 8 * M * N * K}
    return {"bytes": e * (M * K + 2 * N * K + M * N * (3 if c["keep"] else 1)) + vector, "flops": 4 * M * N * K}


# ---- in 64 bits, by other ways than the plain forms ----------------------------------------------------------------
def _act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return torch.where(z > 0, z, torch.zeros_like(z)) if act == "relu" else z.clone()


def _affine64(x, w, b):
    z = torch.matmul(x.double(), w.double().transpose(0, 1))
    return z if b is None else z + b.double()


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "norm":
        x = s["x"].double().requires_grad_(True)
        gamma = s["gamma"].double().requires_grad_(True)
        beta = torch.zeros_like(gamma) if s["beta"] is None else s["beta"].double()
        beta.requires_grad_(True)
        # E x^2 - (E x)^2 is exact enough in 64 bits
        mean = x.mean(-1, keepdim=True) if c["kind"] == "layer" else torch.zeros_like(x[:, :1])
        rstd = (x.square().mean(-1, keepdim=True) - mean.square() + EPS).pow(-0.5)
        y = (x - mean) * (rstd * gamma) + beta
        if c["direction"] == "fwd":
            o = {"y": y.detach(), "rstd": rstd.detach()[:, 0]}
            return {**o, "mean": mean.detach()[:, 0]} if c["kind"] == "layer" else o
        dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), s["dy"].double())
        o = {"dx": dx if s["d_residual"] is None else dx + s["d_residual"].double(), "dgamma": dgamma}
        return {**o, "dbeta": dbeta} if c["kind"] == "layer" else o
    if c["op"] == "linear":
        if c["direction"] == "fwd":
            z = _affine64(s["x"], s["w"], s["bias"])
            y = _act64(z, c["act"])
            o = {"y": y if s["residual"] is None else y + s["residual"].double()}
            return {**o, "z": z} if c["keep"] else o
        dz = s["dy"].double()
        if c["act"] != "none":
            z = s["z"].double().requires_grad_(True)
            dz, = torch.autograd.grad(_act64(z, c["act"]), z, dz)
        o = {"dx": torch.matmul(dz, s["w"].double()), "dw": torch.matmul(dz.transpose(0, 1), s["x"].double())}
        return {**o, "db": dz.sum(0)} if c["bias"] else o
    if c["direction"] == "fwd":
        a, u = _affine64(s["x"], s["w_gate"], s["b_gate"]), _affine64(s["x"], s["w_up"], s["b_up"])
        o = {"h": _act64(a, c["act"]) * u}
        return {**o, "a": a, "u": u} if c["keep"] else o
    a, u = s["a"].double().requires_grad_(True), s["u"].double().requires_grad_(True)
    da, du = torch.autograd.grad(_act64(a, c["act"]) * u, (a, u), s["dh"].double())
    del a, u
    xd = s["x"].double()
    o = {"dx": torch.matmul(da, s["w_gate"].double()) + torch.matmul(du, s["w_up"].double()),
         "dw_gate": torch.matmul(da.transpose(0, 1), xd), "dw_up": torch.matmul(du.transpose(0, 1), xd)}
    return {**o, "db_gate": da.sum(0), "db_up": du.sum(0)} if c["bias"] else o
