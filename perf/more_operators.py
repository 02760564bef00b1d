"""Performance cases of the residual block in 8 bits: the quantiser of a matrix, the norm that adds the residual and writes 8 bits,
and the products that read them, the linear projection and the gated pair, each forward and backward.

Numbers in 8 bits are e4m3 codes with one power of two for each group of 128: of 128 columns of a row (activations, gradients) or of a
block of 128 x 128 (weights).  With A the largest magnitude of a group its exponent e is the least integer >= -127 with
A <= 448 * 2^e, and a code is the value times 2^-e rounded to e4m3, ties to even.  The scales 2^e of a matrix (R, C) are a tensor of
type e8m0 and shape (ceil(C / 128), R) or (ceil(C / 128), ceil(R / 128)).  What the products leave is bf16.

A case is a dict of plain values: ``op`` and ``direction``, the sizes (M tokens, K input columns, N output columns; the norm has D
columns; the quantised matrix is M x K), the type of what is not in 8 bits, and which of the optional parts are there.  Norm weights,
biases, row statistics and the gradients of vectors are single precision throughout; a backward case is given what the forward
call left, and the weights' transposes in 8 bits, as a training program has them in hand.

4096 columns are those of the 8 heads of 512 that the cell's configurations use, 16384 tokens those of the training configuration (2
sequences of 8192); 10944 is 8/3 of 4096, rounded up to whole blocks of 64.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _quant(name, M, K, rows, plain=True, transposed=True, dtype="bf16"):
    return {"name": name, "op": "quant", "direction": "fwd", "M": M, "K": K, "rows": rows, "plain": plain, "transposed": transposed,
            "dtype": dtype}


def _norm(name, M, D, kind="rms", dtype="bf16", residual=True, keep=False):
    return {"name": name, "op": "norm", "direction": "fwd", "M": M, "D": D, "kind": kind, "dtype": dtype, "residual": residual,
            "keep": keep}


def _linear(name, direction, M, K, N, act="none", bias=True, residual=False, keep=False):
    return {"name": name, "op": "linear", "direction": direction, "M": M, "K": K, "N": N, "act": act, "dtype": "bf16",
            "bias": bias, "residual": residual, "keep": keep}


def _gated(name, direction, M, K, N, act="silu", bias=False, keep=False):
    return {"name": name, "op": "gated", "direction": direction, "M": M, "K": K, "N": N, "act": act, "dtype": "bf16",
            "bias": bias, "keep": keep}


def listed():
    return [
        # a training step's weights of the feed-forward half, as they are and transposed, after each update
        _quant("quant_weights", 10944, 4096, 128),
        # activations in single precision, rows of odd length, for a gradient along the tokens as well
        _quant("quant_ragged_f32", 2999, 1365, 1, dtype="f32"),
        # one token's norm while generating: the smallest call, two per block and token
        _norm("norm_one_token", 1, 4096),
        # the norm of a long prompt: the sum goes on as the residual, the normed rows to the products
        _norm("norm_prompt", 16384, 4096),
        # LayerNorm in single precision with the normed rows kept for training, a width that no vector load divides
        _norm("norm_ragged_f32", 2999, 1365, kind="layer", dtype="f32", keep=True),
        # one token through the projection out of the heads
        _linear("linear_one_token", "fwd", 1, 4096, 4096, residual=True),
        # a prompt of ordinary, odd length through it
        _linear("linear_prompt", "fwd", 2000, 4096, 4096, residual=True),
        # training a projection of that width on one long sequence
        _linear("linear_train", "bwd", 8192, 4096, 4096),
        # four sequences generating together through the wide half of the feed-forward block: weights read once
        _gated("gated_decode", "fwd", 4, 4096, 10944),
        # a long sequence through it, with what the backward pass needs kept
        _gated("gated_train_fwd", "fwd", 8192, 4096, 10944, keep=True),
        # and its backward pass: the largest call
        _gated("gated_train_bwd", "bwd", 8192, 4096, 10944),
        # a small odd one: rows of codes that start at odd addresses, biases, the other activation
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
    return w["bytes"] / 4e12 + w["flops"] / 2e15


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op, direction = rng.choice(["quant", "norm", "linear", "linear", "gated", "gated"]), rng.choice(["fwd", "bwd"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op == "quant":
            t = rng.choice(["plain", "transposed", "both"])
            c = _quant("", _log_int(rng, 1, 16384), _columns(rng, 64, 11008), rng.choice([1, 128]), t != "transposed", t != "plain", dtype)
        elif op == "norm":
            c = _norm("", _log_int(rng, 1, 32768), _columns(rng, 64, 8192), rng.choice(["rms", "rms", "layer"]), dtype, rng.random() < 0.7,
                      rng.random() < 0.3)
        elif op == "linear":
            c = _linear("", direction, _log_int(rng, 1, 16384), _columns(rng, 64, 8192), _columns(rng, 64, 8192),
                        rng.choice(["none", "none", "silu", "gelu", "relu"]), rng.random() < 0.5,
                        direction == "fwd" and rng.random() < 0.5, direction == "fwd" and rng.random() < 0.3)
        else:
            c = _gated("", direction, _log_int(rng, 1, 8192), _columns(rng, 64, 4096), _columns(rng, 64, 10944),
                       rng.choice(["silu", "silu", "gelu", "relu"]), rng.random() < 0.3, direction == "fwd" and rng.random() < 0.5)
        del c["name"]
        if _cost(c) <= most:
            return c


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    c, t, gen = case, _type(case), torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=t):
        return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)

    def stream(M, D):
        # the residual stream: columns of different size, rows that have drifted from zero
        scale = torch.exp(0.5 * torch.randn(D, generator=gen, device="cuda"))
        x = torch.randn((M, D), generator=gen, device="cuda") * scale
        return (x + 0.3 * torch.randn((M, 1), generator=gen, device="cuda")).to(t)

    s = {"case": dict(c), "out": {}}
    M = c["M"]
    if c["op"] == "quant":
        s["x"] = normal(M, c["K"], std=c["K"] ** -0.5) if c["rows"] == 128 else stream(M, c["K"])
        return s
    if c["op"] == "norm":
        D = c["D"]
        s["x"] = stream(M, D)
        s["residual"] = normal(M, D) if c["residual"] else None
        s["gamma"] = normal(D, std=0.2, mean=1.0, dtype=torch.float32)
        s["beta"] = normal(D, std=0.2, dtype=torch.float32) if c["kind"] == "layer" else None
        return s
    K, N, fwd = c["K"], c["N"], c["direction"] == "fwd"
    x = normal(M, K)
    weights = [normal(N, K, std=K ** -0.5, dtype=torch.bfloat16) for _ in range(1 if c["op"] == "linear" else 2)]
    s["bias"] = [normal(N, std=0.1, dtype=torch.float32) if c["bias"] else None for _ in weights]
    # (a forward case has the weights as they are, a backward case their transposes)
    s["w"] = [_quantise(w if fwd else w.t(), 128) for w in weights]
    if fwd:
        s["x"] = _quantise(x, 1)
        s["residual"] = normal(M, N) if c["op"] == "linear" and c["residual"] else None
        return s
    s["x"] = x
    s["dy"] = normal(M, N)
    xf = _values(*_quantise(x, 1))
    z = [(xf @ _values(*w) + (0 if b is None else b)).to(t) for w, b in zip(s["w"], s["bias"])]
    s["z"] = z if c["op"] == "gated" or c["act"] != "none" else [None]
    return s


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    return {"quant": {"fwd": _quant_fwd}, "norm": {"fwd": _norm_fwd}, "linear": {"fwd": _product_fwd, "bwd": _product_bwd},
            "gated": {"fwd": _product_fwd, "bwd": _product_bwd}}[c["op"]][c["direction"]](state, c)


# ---- the framework's calls ------------------------------------------------------------------------------------------
def _run_own(s, c):
    # the program owns its output tensors and workspaces: the first call leaves them in s["out"], later ones write there
    import paper_2503_14376_amd as tfla
    fwd, o = c["direction"] == "fwd", s["out"]
    if c["op"] == "quant":
        tfla.q8_quant(s["x"], rows=c["rows"], want_q=c["plain"], want_t=c["transposed"], out=o)
        return {k: o[k] for k in (("q", "scale") if c["plain"] else ()) + (("qt", "scale_t") if c["transposed"] else ())}
    if c["op"] == "norm":
        layer = c["kind"] == "layer"
        tfla.norm_q8_fwd(s["x"], s["gamma"], s["beta"], s["residual"], norm_kind=tfla.NORM_LAYER if layer else tfla.NORM_RMS, norm_eps=EPS,
                         keep_y=c["keep"], out=o)
        names = ("q", "scale", "rstd") + (("mean",) if layer else ()) + (("sum",) if c["residual"] else ()) + (("y",) if c["keep"] else ())
        return {k: o[k] for k in names}
    act = {"none": tfla.ACT_NONE, "silu": tfla.ACT_SILU, "gelu": tfla.ACT_GELU, "relu": tfla.ACT_RELU}[c["act"]]
    if c["op"] == "linear":
        if fwd:
            tfla.linear_q8_fwd(*s["x"], *s["w"][0], s["bias"][0], s["residual"], act=act, keep_pre=c["keep"], out=o)
            return {k: o[k] for k in (("y", "z") if c["keep"] else ("y",))}
        tfla.linear_q8_bwd(s["x"], *s["w"][0], s["dy"], s["z"][0], act=act, want_db=c["bias"], out=o)
        return {k: o[k] for k in (("dx", "dw", "db") if c["bias"] else ("dx", "dw"))}
    if fwd:
        tfla.gated_q8_fwd(*s["x"], *s["w"][0], *s["w"][1], *s["bias"], act=act, keep_pre=c["keep"], out=o)
        return {k: o[k] for k in (("hq", "h_scale", "h", "a", "u") if c["keep"] else ("hq", "h_scale"))}
    tfla.gated_q8_bwd(s["x"], *s["w"][0], *s["w"][1], *s["z"], s["dy"], act=act, want_db=c["bias"], out=o)
    names = ("dx", "dw_gate", "dw_up") + (("db_gate", "db_up") if c["bias"] else ())
    return {k: o[k] for k in names}


# ---- the plain forms: single precision, rounded once at the end ---------------------------------------------------
def _blocks(x, rows):
    """x (R, C) in float with zeros behind its ends, as (R / rows, rows, C / 128, 128)"""
    R, C = x.shape
    x = torch.nn.functional.pad(x, (0, -C % 128, 0, -R % rows))
    return x.reshape(x.shape[0] // rows, rows, x.shape[1] // 128, 128)


def _quantise(x, rows):
    R, C = x.shape
    b = _blocks(x.float(), rows)
    # A = m 2^k with m in [1/2, 1); 448 = 7/8 2^9
    m, k = torch.frexp(b.abs().amax((1, 3)))
    e = torch.where(m > 0, k - 9 + (m > 0.875), torch.full_like(k, -127)).clamp_min(-127)
    q = torch.ldexp(b, -e[:, None, :, None]).reshape(b.shape[0] * rows, -1)[:R, :C].contiguous().to(E4M3)
    return q, (e + 127).to(torch.uint8).t().contiguous().view(E8M0)


def _values(q, scale):
    """what codes and scales stand for, in float"""
    R, C = q.shape
    rows = 1 if scale.shape[1] == R else 128
    s = scale.view(torch.uint8).t().int() - 127
    b = _blocks(q.float(), rows)
    return torch.ldexp(b, s[:, None, :, None]).reshape(b.shape[0] * rows, -1)[:R, :C]


def _quant_fwd(s, c):
    o = {}
    if c["plain"]:
        o["q"], o["scale"] = _quantise(s["x"], c["rows"])
    if c["transposed"]:
        o["qt"], o["scale_t"] = _quantise(s["x"].t(), c["rows"])
    return o


def _norm_fwd(s, c):
    x, o = s["x"].float(), {}
    if c["residual"]:
        x = x + s["residual"].float()
        o["sum"] = x.to(_type(c))
    if c["kind"] == "layer":
        mean = x.sum(-1, keepdim=True) / c["D"]
        x = x - mean
        o["mean"] = mean[:, 0]
    rstd = 1 / torch.sqrt((x * x).sum(-1, keepdim=True) / c["D"] + EPS)
    y = x * rstd * s["gamma"]
    if s["beta"] is not None:
        y = y + s["beta"]
    o["rstd"] = rstd[:, 0]
    o["q"], o["scale"] = _quantise(y, 1)
    if c["keep"]:
        o["y"] = y.to(_type(c))
    return o


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
    return (z > 0).to(z.dtype)


def _product_fwd(s, c):
    t, x = _type(c), _values(*s["x"])
    z = [x @ _values(*w).t() + (0 if b is None else b) for w, b in zip(s["w"], s["bias"])]
    y = _act(z[0], c["act"])
    if c["op"] == "linear":
        if s["residual"] is not None:
            y = y + s["residual"].float()
        o = {"y": y.to(t)}
        if c["keep"]:
            o["z"] = z[0].to(t)
        return o
    h = y * z[1]
    q, scale = _quantise(h, 1)
    o = {"hq": q, "h_scale": scale}
    if c["keep"]:
        o["h"], o["a"], o["u"] = h.to(t), z[0].to(t), z[1].to(t)
    return o


def _product_bwd(s, c):
    t, dy, z = _type(c), s["dy"].float(), s["z"]
    if c["op"] == "linear":
        dz = [dy if z[0] is None else dy * _act_grad(z[0].float(), c["act"])]
        names = ("",)
    else:
        a, u = z[0].float(), z[1].float()
        dz = [dy * u * _act_grad(a, c["act"]), dy * _act(a, c["act"])]
        names = ("_gate", "_up")
    # products in 8 bits: of dz along its columns with the weights, of dz and x along the tokens
    xt = _values(*_quantise(s["x"].t(), 1))
    dx = _values(*_quantise(dz[0], 1)) @ _values(*s["w"][0]).t()
    if c["op"] == "gated":
        dx = dx + _values(*_quantise(dz[1], 1)) @ _values(*s["w"][1]).t()
    o = {"dx": dx.to(t)}
    o.update(("dw" + n, (_values(*_quantise(d.t(), 1)) @ xt.t()).to(t)) for n, d in zip(names, dz))
    if c["bias"]:
        o.update(("db" + n, d.sum(0)) for n, d in zip(names, dz))
    return o


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    c = case
    e, M, up = (2 if c["dtype"] == "bf16" else 4), c["M"], lambda n: -(-n // 128)
    if c["op"] == "quant":
        K, copies = c["K"], c["plain"] + c["transposed"]
        scales = (c["plain"] * up(K) * M + c["transposed"] * up(M) * K) if c["rows"] == 1 else copies * up(K) * up(M)
        return {"bytes": M * K * (e + copies) + scales, "flops": M * K * 2 * copies}
    if c["op"] == "norm":
        D, layer = c["D"], c["kind"] == "layer"
        tensors = 1 + 2 * c["residual"] + c["keep"]
        vectors = 4 * M * (2 if layer else 1) + 4 * D * (2 if layer else 1)
        return {"bytes": tensors * M * D * e + M * D + up(D) * M + vectors, "flops": M * D * 10}
    K, N, pair = c["K"], c["N"], 2 if c["op"] == "gated" else 1
    weights, vector = pair * (N * K + up(N) * up(K)), 4 * N * pair if c["bias"] else 0
    if c["direction"] == "fwd":
        x = M * K + up(K) * M
        if pair == 1:
            return {"bytes": x + weights + e * M * N * (1 + c["residual"] + c["keep"]) + vector, "flops": 2 * M * N * K}
        return {"bytes": x + weights + M * N + up(N) * M + e * M * N * (3 if c["keep"] else 0) + vector, "flops": 4 * M * N * K}
    mn = 3 if pair == 2 else 1 + (c["act"] != "none")
    return {"bytes": weights + e * (2 * M * K + pair * N * K + mn * M * N) + vector, "flops": 4 * pair * M * N * K}


# ---- in 64 bits, by other ways than the plain forms ----------------------------------------------------------------
def _round64(v):
    """to the nearest e4m3 value, ties to even: steps of 2^-3 of the power of two below, of 2^-9 below 2^-6"""
    p = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -30)))
    p = torch.where(torch.exp2(p + 1) <= v.abs(), p + 1, torch.where(torch.exp2(p) > v.abs(), p - 1, p))
    step = torch.exp2(p.clamp_min(-6) - 3)
    return torch.round(v / step) * step


def _coded64(x, along, across=1):
    """codes (as values) and scales of x in groups of `along` columns and `across` rows, rows x blocks"""
    R, C = x.shape
    full = x.new_zeros((-(-R // across) * across, -(-C // along) * along))
    full[:R, :C] = x
    most = full.abs().reshape(-1, across, full.shape[1]).amax(1).reshape(-1, full.shape[1] // along, along).amax(2)
    e = torch.ceil(torch.log2(most.clamp_min(2.0 ** -140) / 448))
    e = e + (most > 448 * torch.exp2(e)) - (most <= 448 * torch.exp2(e - 1)).to(e.dtype)
    scale = torch.exp2(e.clamp_min(-127))
    wide = scale.repeat_interleave(across, 0).repeat_interleave(along, 1)[:R, :C]
    return _round64(x / wide), scale, wide


def _stand64(q, scale):
    """what given codes and scales stand for"""
    s = torch.exp2(scale.view(torch.uint8).double() - 127).transpose(0, 1)
    if s.shape[0] != q.shape[0]:
        s = s.repeat_interleave(128, 0)[:q.shape[0]]
    return q.double() * s.repeat_interleave(128, 1)[:, :q.shape[1]]


def _requant64(x):
    q, _, wide = _coded64(x, 128)
    return q * wide


def _act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return torch.where(z > 0, z, torch.zeros_like(z)) if act == "relu" else z.clone()


def exact(case, seed):
    # Codes and scales of given values have one exact value.  Those of values that a call itself computes have none: next to a border
    # between two codes, or two powers of two, the last bit of a sum in 32 bits tells the side (the values are checked where they are kept).
    s, c = prepare(case, seed), case
    if c["op"] == "quant":
        x, o = s["x"].double(), {}
        if c["plain"]:
            q, scale, _ = _coded64(x, 128, c["rows"])
            o["q"], o["scale"] = q, scale.transpose(0, 1).contiguous()
        if c["transposed"]:
            q, scale, _ = _coded64(x.transpose(0, 1), 128, c["rows"])
            o["qt"], o["scale_t"] = q, scale.transpose(0, 1).contiguous()
        return o
    if c["op"] == "norm":
        x = s["x"].double()
        o = {}
        if c["residual"]:
            o["sum"] = x = x + s["residual"].double()
        # E x^2 - (E x)^2 is exact enough in 64 bits
        mean = x.mean(-1, keepdim=True) if c["kind"] == "layer" else torch.zeros_like(x[:, :1])
        rstd = (x.square().mean(-1, keepdim=True) - mean.square() + EPS).pow(-0.5)
        y = (x - mean) * (rstd * s["gamma"].double())
        if s["beta"] is not None:
            y = y + s["beta"].double()
        o.update(q=None, scale=None, rstd=rstd[:, 0])
        if c["kind"] == "layer":
            o["mean"] = mean[:, 0]
        if c["keep"]:
            o["y"] = y
        return o
    bias = [0.0 if b is None else b.double() for b in s["bias"]]
    if c["direction"] == "fwd":
        x = _stand64(*s["x"])
        z = [torch.matmul(x, _stand64(*w).transpose(0, 1)) + b for w, b in zip(s["w"], bias)]
        if c["op"] == "linear":
            y = _act64(z[0], c["act"])
            o = {"y": y if s["residual"] is None else y + s["residual"].double()}
            return {**o, "z": z[0]} if c["keep"] else o
        h = _act64(z[0], c["act"]) * z[1]
        o = {"hq": None, "h_scale": None}
        return {**o, "h": h, "a": z[0], "u": z[1]} if c["keep"] else None
    dz = [s["dy"].double()]
    if c["op"] == "gated":
        a, u = (z.double().requires_grad_(True) for z in s["z"])
        dz = list(torch.autograd.grad(_act64(a, c["act"]) * u, (a, u), dz[0]))
        del a, u
    elif c["act"] != "none":
        z = s["z"][0].double().requires_grad_(True)
        dz = list(torch.autograd.grad(_act64(z, c["act"]), z, dz[0]))
    names = ("_gate", "_up") if c["op"] == "gated" else ("",)
    xt = _requant64(s["x"].double().transpose(0, 1))
    o = {"dx": sum(torch.matmul(_requant64(d), _stand64(*w).transpose(0, 1)) for d, w in zip(dz, s["w"]))}
    o.update(("dw" + n, torch.matmul(_requant64(d.transpose(0, 1)), xt.transpose(0, 1))) for n, d in zip(names, dz))
    if c["bias"]:
        o.update(("db" + n, d.sum(0)) for n, d in zip(names, dz))
    return o
