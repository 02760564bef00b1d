"""Every kernel of the residual block's products at the sizes of tests/block_sizes.py, against 64-bit forms: outputs at odd addresses between
bytes of a known pattern, a workspace of exactly the size that the query returns, filled with NaN, between such bytes too."""
import pytest
import torch

from tests import block_util as bu
from tests.block_sizes import SIZES
from tests.test_gpu_block import ACTS, BF16, F32, code, fenced, generator, normal

pytestmark = pytest.mark.gpu
PATTERN, AROUND = 0x5B, 4096


@pytest.fixture(scope="module")
def tfla():
    import paper_2503_14376_amd as pkg
    pkg.load_library()
    return pkg


class Fences:
    """tensors inside larger allocations of PATTERN, which intact() looks for again"""

    def __init__(self):
        self.edges = []

    def _inside(self, size, at):
        buf = torch.full((size + at + AROUND,), PATTERN, dtype=torch.uint8, device="cuda")
        self.edges += [buf[:at], buf[at + size:]]
        return buf[at:at + size]

    def tensor(self, shape, dtype, shift):
        size = torch.empty(0, dtype=dtype).element_size()
        n = 1
        for d in shape:
            n *= d
        return self._inside(n * size, AROUND + shift * size).view(dtype).view(shape)

    def workspace(self, size):
        return None if size == 0 else self._inside(size, AROUND).fill_(0xFF)      # (NaN in either type)

    def intact(self):
        for i, e in enumerate(self.edges):
            assert bool((e == PATTERN).all()), ("before" if i % 2 == 0 else "behind", "tensor", i // 2)


def outputs(fences, shift, dtype, M=0, **shapes):
    return {k: fences.tensor(s, F32 if k.startswith(("db", "rstd", "mean", "dg")) else dtype, shift) for k, s in shapes.items()}


def label(case):
    b, d, p, M, K, N = case
    return "%s-%s-%s-%dx%dx%d" % ("bwd" if b else "fwd", "bf16" if d else "fp32", "pair" if p else "one", M, K, N)


@pytest.mark.parametrize("i", range(len(SIZES)), ids=[label(c) for c in SIZES])
def test_product(tfla, i):
    backward, b16, pair, M, K, N = SIZES[i]
    print(label(SIZES[i]), flush=True)
    dtype, shift = BF16 if b16 else F32, i % 3
    act = ACTS[i % 4]
    gen, fences = generator(i), Fences()
    query = tfla.gated_workspace_bytes if pair else tfla.linear_workspace_bytes
    need = query(backward, M, K, N, code(tfla, act), tfla.BF16 if b16 else tfla.F32)
    kw = dict(act=code(tfla, act))
    x = fenced(normal(gen, M, K, dtype=dtype))
    w, w2 = (fenced(normal(gen, N, K, std=K ** -0.5, dtype=dtype)) for _ in range(2))
    b, r = fenced(normal(gen, N, std=0.3), shift), fenced(normal(gen, M, N, dtype=dtype), shift)
    if not backward and pair:
        o = outputs(fences, shift, dtype, h=(M, N), a=(M, N), u=(M, N))
        tfla.gated_fwd(x, w, w2, b, None, keep_pre=True, workspace=fences.workspace(need), out=o, **kw)
        for name, ref in zip("auh", bu.gated(x, w, w2, b, None, act)):
            bu.within(name, o[name], *ref)
        lean = outputs(fences, shift, dtype, h=(M, N))
        tfla.gated_fwd(x, w, w2, b, None, workspace=fences.workspace(need), out=lean, **kw)
        assert torch.equal(lean["h"], o["h"])
    elif not backward:
        o = outputs(fences, shift, dtype, y=(M, N), z=(M, N))
        tfla.linear_fwd(x, w, b, r, keep_pre=True, workspace=fences.workspace(need), out=o, **kw)
        z, y = bu.linear(x, w, b, r, act)
        bu.within("z", o["z"], *z)
        bu.within("y", o["y"], *y)
        # the result in the place of the residual, without z
        same = outputs(fences, shift, dtype, y=(M, N))
        same["y"].copy_(r)
        tfla.linear_fwd(x, w, b, same["y"], workspace=fences.workspace(need), out=same, **kw)
        assert torch.equal(same["y"], o["y"])
    elif pair:
        o = outputs(fences, shift, dtype, dx=(M, K), dw_gate=(N, K), dw_up=(N, K), db_gate=(N,), db_up=(N,))
        a, u, dh = (fenced(normal(gen, M, N, dtype=dtype)) for _ in range(3))
        tfla.gated_bwd(x, w, w2, a, u, dh, want_db=True, workspace=fences.workspace(need), out=o, **kw)
        av, uv, d = a.to(bu.F64), u.to(bu.F64), dh.to(bu.F64)
        da, du = d * uv * bu.act_grad(av, act), d * bu.act(av, act)
        e = bu.FN * (1 + av.abs()) * d.abs()
        dx, dw, db = bu.back([da, du], [e * uv.abs() + bu.U * da.abs(), e + bu.U * du.abs()], x, [w, w2], dtype)
        for name, ref in (("dx", dx), ("dw_gate", dw[0]), ("dw_up", dw[1]), ("db_gate", db[0]), ("db_up", db[1])):
            bu.within(name, o[name], *ref)
    else:
        o = outputs(fences, shift, dtype, dx=(M, K), dw=(N, K), db=(N,))
        z, dy = (fenced(normal(gen, M, N, dtype=dtype)) for _ in range(2))
        tfla.linear_bwd(x, w, dy, z, want_db=True, workspace=fences.workspace(need), out=o, **kw)
        d = dy.to(bu.F64)
        dz = d * bu.act_grad(z.to(bu.F64), act)
        e = torch.zeros_like(dz) if act == "none" else bu.FN * d.abs() * (1 + z.to(bu.F64).abs())
        dx, dw, db = bu.back([dz], [e], x, [w], dtype)
        for name, ref in (("dx", dx), ("dw", dw[0]), ("db", db[0])):
            bu.within(name, o[name], *ref)
    fences.intact()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,D", [(1, 1), (3, 7), (2, 511), (9, 512), (5, 777), (33, 1024), (40, 1365), (9, 2049), (700, 4096), (6, 4104), (3, 8191),
                                 (2, 10000), (600, 100)])
def test_norm_between_fences(tfla, dtype, M, D):
    print("norm", M, D, dtype, flush=True)
    gen, fences, shift = generator(M + D), Fences(), (M + D) % 3
    x, dy, res = (fenced(normal(gen, M, D, dtype=dtype), shift) for _ in range(3))
    gamma, beta = (fenced(normal(gen, D), shift) for _ in range(2))
    o = outputs(fences, shift, dtype, y=(M, D), rstd=(M,), mean=(M,))
    tfla.norm_fwd(x, gamma, beta, norm_kind=tfla.NORM_LAYER, norm_eps=1e-5, out=o)
    mean, rstd, y = bu.norm(x, gamma, beta, True, 1e-5)
    bu.within("mean", o["mean"], *mean)
    if D > 1:                 # (a row of one value has no variance: rstd is eps's alone)
        bu.within("rstd", o["rstd"], *rstd)
    bu.within("y", o["y"], *y)
    g = outputs(fences, shift, dtype, dx=(M, D), dgamma=(D,), dbeta=(D,))
    need = tfla.norm_workspace_bytes(1, M, D, tfla.BF16 if dtype == BF16 else tfla.F32, tfla.NORM_LAYER)
    tfla.norm_bwd(x, dy, o["rstd"], o["mean"], gamma, res, norm_kind=tfla.NORM_LAYER, want_dbeta=True, workspace=fences.workspace(need), out=g)
    for name, ref in zip(("dx", "dgamma", "dbeta"), bu.norm_back(x, dy, o["rstd"], o["mean"], gamma, res, True)):
        bu.within(name, g[name], *ref)
    fences.intact()


@pytest.mark.parametrize("shifts", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 2, 1)])
@pytest.mark.parametrize("M,K,N", [(3, 72, 70), (40, 128, 264), (300, 264, 136), (270, 333, 129)])
@pytest.mark.parametrize("pair", [False, True])
def test_workspaces_of_copied_operands(tfla, shifts, M, K, N, pair):
    """bf16 operands off 16 bytes, each alone: copies into a workspace of the size that the query names for them"""
    print("copied", shifts, M, K, N, pair, flush=True)
    gen, fences = generator(M), Fences()
    x, w, w2 = (fenced(normal(gen, r, K, std=K ** -0.5, dtype=BF16), s) for r, s in ((M, shifts[0]), (N, shifts[1]), (N, shifts[1])))
    a, u, dy = (fenced(normal(gen, M, N, dtype=BF16), s) for s in (0, 0, shifts[2]))
    query = tfla.gated_workspace_bytes if pair else tfla.linear_workspace_bytes
    need = [query(b, M, K, N, tfla.ACT_NONE, tfla.BF16, True) for b in (0, 1)]
    kw = dict(act=tfla.ACT_NONE)
    if pair:
        o, g = outputs(fences, 1, BF16, h=(M, N)), outputs(fences, 1, BF16, dx=(M, K), dw_gate=(N, K), dw_up=(N, K))
        tfla.gated_fwd(x, w, w2, workspace=fences.workspace(need[0]), out=o, **kw)
        bu.within("h", o["h"], *bu.gated(x, w, w2, None, None, "none")[2])
        tfla.gated_bwd(x, w, w2, a, u, dy, workspace=fences.workspace(need[1]), out=g, **kw)
        d = [dy.to(bu.F64) * u.to(bu.F64), dy.to(bu.F64) * a.to(bu.F64)]
        dx, dw, _ = bu.back(d, [bu.U * t.abs() for t in d], x, [w, w2], BF16)
    else:
        o, g = outputs(fences, 1, BF16, y=(M, N)), outputs(fences, 1, BF16, dx=(M, K), dw=(N, K))
        tfla.linear_fwd(x, w, workspace=fences.workspace(need[0]), out=o, **kw)
        bu.within("y", o["y"], *bu.linear(x, w, None, None, "none")[1])
        tfla.linear_bwd(x, w, dy, workspace=fences.workspace(need[1]), out=g, **kw)
        dx, dw, _ = bu.back([dy.to(bu.F64)], [torch.zeros_like(dy, dtype=bu.F64)], x, [w], BF16)
    bu.within("dx", g["dx"], *dx)
    for name, ref in zip(("dw_gate", "dw_up") if pair else ("dw",), dw):
        bu.within(name, g[name], *ref)
    fences.intact()
