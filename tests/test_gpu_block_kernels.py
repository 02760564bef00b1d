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
