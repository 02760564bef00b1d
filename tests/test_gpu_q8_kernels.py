"""Every kernel of the products in 8 bits at the sizes of tests/q8_sizes.py, with codes and values whose products add without rounding, so that
results are compared for equality: operands between codes and scales that are NaN, outputs at odd addresses between bytes of a known
pattern, a workspace of exactly the size that the query returns, filled with NaN, between such bytes too."""
import pytest
import torch

from tests import q8_util as ref
from tests.block_util import F64
from tests.q8_util import E4M3, E8M0
from tests.test_gpu_block_kernels import Fences
from tests.q8_sizes import SIZES

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def tfla():
    import paper_2503_14376_amd as pkg
    pkg.load_library()
    return pkg


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def among_nan(t, shift=0):
    """the tensor `shift` elements behind a multiple of 16 bytes, between bytes of 0xFF: NaN as code, scale, bf16 and fp32"""
    size = t.numel() * t.element_size()
    buf = torch.full((size + 8192,), 0xFF, dtype=torch.uint8, device="cuda")
    at = 4096 + shift * t.element_size()
    buf[at:at + size] = t.contiguous().view(torch.uint8).view(-1)
    return buf[at:at + size].view(t.dtype).view(t.shape)


def codes(gen, R, C, rows, shift=0):
    q, s = ref.small_codes(gen, R, C, rows)
    return among_nan(q, shift), among_nan(s, shift)


def values(gen, R, C, most=2, shift=0):
    """0, +-1, ..., +-2^most: codes stand for them exactly, and sums of products are exact"""
    v = torch.exp2(torch.randint(0, most + 1, (R, C), generator=gen, device="cuda").float())
    return among_nan((v * torch.randint(-1, 2, (R, C), generator=gen, device="cuda")).to(BF16), shift)


def rounded(x):
    return x.float().to(BF16)


def outputs(fences, shift, **shapes):
    kind = {"hq": E4M3, "q": E4M3, "qt": E4M3, "h_scale": E8M0, "scale": E8M0, "scale_t": E8M0}
    return {k: fences.tensor(s, kind.get(k, F32 if k.startswith("db") else BF16), shift) for k, s in shapes.items()}


def forward(tfla, gen, pair, M, K, N, shift, off=(0, 0)):
    fences = Fences()
    x, w, w2 = codes(gen, M, K, 1, off[0]), codes(gen, N, K, 128, off[1]), codes(gen, N, K, 128, off[1])
    query = tfla.gated_q8_workspace_bytes if pair else tfla.linear_q8_workspace_bytes
    need = query(0, M, K, N, tfla.ACT_RELU, any(off))
    a = ref.stands(*x) @ ref.stands(*w).t()
    bias = among_nan(torch.randint(-8, 9, (N,), generator=gen, device="cuda").float(), shift)
    if pair:
        a, u = a + bias, ref.stands(*x) @ ref.stands(*w2).t()
        h = a.clamp_min(0).float() * u.float()                  # (one rounding in fp32)
        o = outputs(fences, shift, hq=(M, N), h_scale=(-(-N // 128), M), h=(M, N), a=(M, N), u=(M, N))
        tfla.gated_q8_fwd(*x, *w, *w2, bias, act=tfla.ACT_RELU, keep_pre=True, workspace=fences.workspace(need), out=o)
        assert torch.equal(o["a"], rounded(a)) and torch.equal(o["u"], rounded(u)) and torch.equal(o["h"], h.to(BF16))
        ref.same_codes(o["hq"], o["h_scale"], *ref.quant(h), "h")
        lean = outputs(fences, shift, hq=(M, N), h_scale=(-(-N // 128), M))
        tfla.gated_q8_fwd(*x, *w, *w2, bias, act=tfla.ACT_RELU, workspace=fences.workspace(need), out=lean)
        for k in lean:
            assert k == "workspace" or torch.equal(lean[k].view(torch.uint8), o[k].view(torch.uint8)), k
    else:
        z = a + bias
        r = among_nan(torch.randint(-8, 9, (M, N), generator=gen, device="cuda").to(BF16), shift)
        o = outputs(fences, shift, y=(M, N), z=(M, N))
        tfla.linear_q8_fwd(*x, *w, bias, r, act=tfla.ACT_RELU, keep_pre=True, workspace=fences.workspace(need), out=o)
        assert torch.equal(o["z"], rounded(z)) and torch.equal(o["y"], rounded(z.clamp_min(0) + r.to(F64)))
        # the result in the place of the residual, without z
        same = outputs(fences, shift, y=(M, N))
        same["y"].copy_(r)
        tfla.linear_q8_fwd(*x, *w, bias, same["y"], act=tfla.ACT_RELU, workspace=fences.workspace(need), out=same)
        assert torch.equal(same["y"], o["y"])
    fences.intact()


def backward(tfla, gen, pair, M, K, N, shift, off=0):
    fences = Fences()
    x, dy = values(gen, M, K, 1, shift), values(gen, M, N, 1, shift)
    ws = [values(gen, N, K, 1) for _ in range(2 if pair else 1)]
    wt = [tfla.q8_quant(w, rows=128, want_q=False, want_t=True) for w in ws]
    wt = [(among_nan(t["qt"], off), among_nan(t["scale_t"], off)) for t in wt]
    z, u = values(gen, M, N, 1, shift), values(gen, M, N, 1, shift)
    query = tfla.gated_q8_workspace_bytes if pair else tfla.linear_q8_workspace_bytes
    need = query(1, M, K, N, tfla.ACT_RELU, off != 0)
    d, zd = dy.to(F64), z.to(F64)
    if pair:
        o = outputs(fences, shift, dx=(M, K), dw_gate=(N, K), dw_up=(N, K), db_gate=(N,), db_up=(N,))
        tfla.gated_q8_bwd(x, *wt[0], *wt[1], z, u, dy, act=tfla.ACT_RELU, want_db=True, workspace=fences.workspace(need), out=o)
        dz, names = [d * u.to(F64) * (zd > 0), d * zd.clamp_min(0)], ("_gate", "_up")
    else:
        o = outputs(fences, shift, dx=(M, K), dw=(N, K), db=(N,))
        tfla.linear_q8_bwd(x, *wt[0], dy, z, act=tfla.ACT_RELU, want_db=True, workspace=fences.workspace(need), out=o)
        dz, names = [d * (zd > 0)], ("",)
    assert torch.equal(o["dx"], rounded(sum(g @ w.to(F64) for g, w in zip(dz, ws))))
    for n, g in zip(names, dz):
        assert torch.equal(o["dw" + n], rounded(g.t() @ x.to(F64))), n
        assert torch.equal(o["db" + n], g.sum(0).float()), n
    fences.intact()


@pytest.mark.parametrize("i", range(len(SIZES)), ids=["%s-%s-%dx%dx%d" % (("fwd", "bwd")[b], ("one", "pair")[p], *s) for b, p, *s in SIZES])
def test_product(tfla, i):
    back, pair, M, K, N = SIZES[i]
    print(SIZES[i], flush=True)
    (backward if back else forward)(tfla, generator(i), pair, M, K, N, i % 3)


@pytest.mark.parametrize("off", [(1, 0), (0, 1), (3, 7), (15, 8)])
@pytest.mark.parametrize("M,K,N", [(3, 144, 70), (20, 128, 264), (40, 272, 136), (270, 333, 129), (300, 640, 520)])
@pytest.mark.parametrize("pair", [False, True])
def test_operands_off_16_bytes(tfla, off, M, K, N, pair):
    """each alone and both: copies into a workspace of the size that the query names for them, or rows read in place"""
    print("off", off, M, K, N, pair, flush=True)
    forward(tfla, generator(M), pair, M, K, N, 1, off)
    if off[1]:
        backward(tfla, generator(N), pair, M, N, K, 1, off[1])


@pytest.mark.parametrize("M", [1, 4, 5, 8, 9, 16, 17, 32])
@pytest.mark.parametrize("K,N,off", [(1, 20, (0, 0)), (2, 7, (1, 3)), (3, 40, (2, 1)), (5, 33, (0, 2)), (15, 16, (3, 0)), (127, 130, (0, 0)), (129, 64, (0, 1)),
                                     (333, 70, (2, 0)), (1365, 129, (0, 0)), (2049, 140, (5, 2)), (4099, 24, (0, 0)), (4096, 24, (1, 2))])
@pytest.mark.parametrize("pair", [False, True])
def test_few_rows_at_odd_addresses(tfla, M, K, N, off, pair):
    """the first and last words of a row hold bytes of its neighbours or of nothing"""
    print("odd", M, K, N, off, pair, flush=True)
    forward(tfla, generator(M * K), pair, M, K, N, 1, off)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K", [(1, 5), (7, 7), (128, 128), (130, 1365), (300, 264), (129, 8)])
def test_quantiser_between_fences(tfla, M, K, dtype, rows):
    print("quantiser", M, K, dtype, rows, flush=True)
    fences, shift = Fences(), (M + K) % 3
    x = among_nan((torch.randn((M, K), generator=generator(M), device="cuda") * 3).to(dtype), shift)
    o = outputs(fences, shift, q=(M, K), scale=(-(-K // 128), -(-M // rows)), qt=(K, M), scale_t=(-(-M // 128), -(-K // rows)))
    tfla.q8_quant(x, rows=rows, want_t=True, out=o)
    ref.same_codes(o["q"], o["scale"], *ref.quant(x, rows))
    ref.same_codes(o["qt"], o["scale_t"], *ref.quant(x.t().contiguous(), rows))
    fences.intact()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,D", [(1, 1), (3, 7), (9, 512), (5, 777), (40, 1365), (9, 2049), (700, 4096), (6, 4104), (3, 8191), (2, 10000)])
def test_norm_between_fences(tfla, dtype, M, D):
    print("norm", M, D, dtype, flush=True)
    gen, fences, shift = generator(M + D), Fences(), (M + D) % 3
    x, r = (among_nan(torch.randn((M, D), generator=gen, device="cuda").to(dtype), shift) for _ in range(2))
    gamma, beta = (among_nan(torch.randn(D, generator=gen, device="cuda"), shift) for _ in range(2))
    o = outputs(fences, shift, q=(M, D), scale=(-(-D // 128), M))
    o.update({k: fences.tensor(s, t, shift) for k, s, t in (("rstd", (M,), F32), ("mean", (M,), F32), ("sum", (M, D), dtype), ("y", (M, D), dtype))})
    tfla.norm_q8_fwd(x, gamma, beta, r, norm_kind=tfla.NORM_LAYER, keep_y=True, out=o)
    want = tfla.norm_q8_fwd(x.float(), gamma, beta, r.float(), norm_kind=tfla.NORM_LAYER, keep_y=True)
    ref.same_codes(o["q"], o["scale"], *ref.quant(want["y"]))
    assert torch.equal(o["y"], want["y"].to(dtype)) and torch.equal(o["sum"], (x.float() + r.float()).to(dtype))
    fences.intact()
