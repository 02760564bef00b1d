"""The entry points in 8 bits as they are used: one after another, on streams, in captured graphs, with memory that is kept, on values that
are not finite; and the example."""
import importlib.util
import os

import pytest
import torch

from tests import q8_util as ref
from tests.block_util import F64, norm as norm64, within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def tfla():
    import paper_2503_14376_amd as pkg
    pkg.load_library()
    return pkg


def normal(gen, *shape, std=1.0, dtype=BF16):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class FeedForward:
    """norm of x + residual -> gated pair -> projection back plus the sum, forward and backward; outputs and workspaces are kept"""

    def __init__(self, tfla, M, D, F, seed):
        gen = generator(seed)
        self.t, self.M = tfla, M
        self.x, self.r, self.dy = (normal(gen, M, D) for _ in range(3))
        self.gamma = normal(gen, D, dtype=F32)
        self.q = [tfla.q8_quant(w, rows=128, want_t=True) for w in (normal(gen, F, D, std=D ** -0.5), normal(gen, F, D, std=D ** -0.5),
                                                                    normal(gen, D, F, std=F ** -0.5))]
        self.out = [dict() for _ in range(6)]

    def forward(self, keep=False, **kw):
        t, o = self.t, self.out
        g, u, d = ((w["q"], w["scale"]) for w in self.q)
        n = t.norm_q8_fwd(self.x, self.gamma, residual=self.r, keep_y=keep, out=o[0], **kw)
        h = t.gated_q8_fwd(n["q"], n["scale"], *g, *u, keep_pre=keep, out=o[1], **kw)
        return t.linear_q8_fwd(h["hq"], h["h_scale"], *d, residual=n["sum"], out=o[2], **kw)["y"]

    def backward(self, **kw):
        t, o = self.t, self.out
        g, u, d = ((w["qt"], w["scale_t"]) for w in self.q)
        n, h = o[0], o[1]
        down = t.linear_q8_bwd(h["h"], *d, self.dy, out=o[3], **kw)
        pair = t.gated_q8_bwd(n["y"], *g, *u, h["a"], h["u"], down["dx"], out=o[4], **kw)
        back = t.norm_bwd(n["sum"], pair["dx"], n["rstd"], gamma=self.gamma, d_residual=self.dy, out=o[5], **kw)
        return {"dx": back["dx"], "dgamma": back["dgamma"], "dw_down": down["dw"], "dw_gate": pair["dw_gate"], "dw_up": pair["dw_up"]}


@pytest.mark.parametrize("M,D,F", [(1, 256, 704), (4, 512, 1365), (40, 264, 520), (300, 512, 1365)])
def test_one_after_another(tfla, M, D, F):
    """each step from what the one before it left, and the whole against a block in 64 bits within what 8 bits cost"""
    print("together", M, D, F, flush=True)
    b = FeedForward(tfla, M, D, F, M)
    y = b.forward(keep=True)
    n, h = b.out[0], b.out[1]
    _, (rstd, er), (ny, en) = norm64(n["sum"], b.gamma, None, False, 1e-6)
    # (the norm is of the unrounded sum: half a step of bf16 of its terms, in the statistics and in the row)
    half = 2.0 ** -8
    within("y", n["y"], ny, en + 2 * half * (ny.abs() + (n["sum"].to(F64).abs() * rstd[:, None] * b.gamma.to(F64).abs())))
    g, u, d = ((w["q"], w["scale"]) for w in b.q)
    (a, ea), (v, ev), (hh, eh) = ref.gated(ref.stands(n["q"], n["scale"]), ref.stands(*g), ref.stands(*u), None, None, "silu")
    within("h", h["h"], hh, eh)
    ref.coded("hq", h["hq"], h["h_scale"], hh, eh)
    _, (yy, ey) = ref.linear(ref.stands(h["hq"], h["h_scale"]), ref.stands(*d), None, n["sum"], "none")
    within("out", y, yy, ey)
    gr = b.backward()
    (dx, edx), dws, _ = ref.back([b.dy.to(F64)], [torch.zeros(M, D, dtype=F64, device="cuda")], h["h"], [ref.stands(*d)])
    within("dh", b.out[3]["dx"], dx, edx)
    within("dw_down", gr["dw_down"], *dws[0])
    dz, ez = ref.gradients("silu", b.out[3]["dx"], h["a"], h["u"])
    # (codes of the transposed weights stand for what those of the weights do)
    for w, q in zip(b.q, (g, u, d)):
        assert torch.equal(ref.stands(w["qt"], w["scale_t"]), ref.stands(*q).t())
    (dx, edx), dws, _ = ref.back(dz, ez, n["y"], [ref.stands(*g), ref.stands(*u)])
    within("dn", b.out[4]["dx"], dx, edx)
    within("dw_gate", gr["dw_gate"], *dws[0])
    within("dw_up", gr["dw_up"], *dws[1])


@pytest.mark.parametrize("M,D,F", [(1, 256, 704), (130, 512, 1365), (700, 1024, 2752)])
def test_captured_and_replayed(tfla, M, D, F):
    """forward and backward in one graph, replayed on changing inputs between eager calls of another block: bits as without a graph"""
    print("graph", M, D, F, flush=True)
    b, other = FeedForward(tfla, M, D, F, 3), FeedForward(tfla, M, D, F, 4)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b.forward(keep=True); b.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = b.forward(keep=True)
        grads = b.backward()
    for i in range(4):
        gen = generator(100 + i)
        x, dy = normal(gen, M, D), normal(gen, M, D)
        b.x.copy_(x); b.dy.copy_(dy)
        graph.replay()
        other.x.copy_(x); other.r.copy_(b.r); other.dy.copy_(dy); other.gamma.copy_(b.gamma); other.q = b.q
        want_y = other.forward(keep=True)
        want = other.backward()
        torch.cuda.synchronize()
        assert torch.equal(y, want_y), i
        for k in want:
            assert torch.equal(grads[k], want[k]), (i, k)


def test_two_streams_at_once(tfla):
    """two blocks on streams of their own, each with its own outputs and workspaces"""
    print("streams", flush=True)
    blocks = [FeedForward(tfla, 513, 512, 1365, s) for s in (5, 6)]
    want = []
    for b in blocks:
        y = b.forward(keep=True).clone()
        want.append((y, {k: v.clone() for k, v in b.backward().items()}))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(3):
        got = []
        for b, s in zip(blocks, streams):
            b.out = [dict() for _ in range(6)]
            got.append((b.forward(keep=True, stream=s), b.backward(stream=s)))
        torch.cuda.synchronize()
        for (y, g), (wy, wg) in zip(got, want):
            assert torch.equal(y, wy) and all(torch.equal(g[k], wg[k]) for k in wg)


@pytest.mark.parametrize("M,K,N", [(1, 4096, 300), (8, 257, 200), (64, 1024, 64), (300, 1000, 333), (513, 2048, 520), (4100, 2600, 2000),
                                   (40, 4096, 256), (8192, 256, 4096), (4096, 256, 1152)])
def test_a_projection_may_write_over_its_residual(tfla, M, K, N):
    print("in place", M, K, N, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(M + K + N)
    x, w, r = (torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16) for s in ((M, K), (N, K), (M, N)))
    xq, wq = tfla.q8_quant(x), tfla.q8_quant(w, rows=128)
    args = xq["q"], xq["scale"], wq["q"], wq["scale"]
    want = tfla.linear_q8_fwd(*args, residual=r, act=tfla.ACT_SILU)["y"]
    assert tfla.linear_q8_fwd(*args, residual=r, act=tfla.ACT_SILU, out={"y": r})["y"] is r
    assert torch.equal(r.view(torch.int16), want.view(torch.int16))


def test_the_same_call_gives_the_same_bits(tfla):
    print("bits", flush=True)
    b = FeedForward(tfla, 333, 1024, 1365, 7)
    y = b.forward(keep=True).clone()
    g = {k: v.clone() for k, v in b.backward().items()}
    for _ in range(5):
        assert torch.equal(b.forward(keep=True), y)
        assert all(torch.equal(v, g[k]) for k, v in b.backward().items())


@pytest.mark.parametrize("M", [3, 40, 300])
def test_what_is_not_finite_stays_in_its_row(tfla, M):
    """NaN and infinities become the code NaN, a row of a product with one is NaN, others are what they were"""
    print("not finite", M, flush=True)
    gen = generator(M)
    x, w, dy = normal(gen, M, 300), normal(gen, 200, 300, std=0.1), normal(gen, M, 200)
    wq = tfla.q8_quant(w, rows=128, want_t=True)
    bad = x.clone()
    bad[1, 5], bad[M - 1, 299] = float("nan"), float("-inf")
    rows = torch.zeros(M, dtype=torch.bool, device="cuda")
    rows[1] = rows[M - 1] = True
    good_q, bad_q = tfla.q8_quant(x), tfla.q8_quant(bad)
    y = tfla.linear_q8_fwd(good_q["q"], good_q["scale"], wq["q"], wq["scale"])["y"]
    z = tfla.linear_q8_fwd(bad_q["q"], bad_q["scale"], wq["q"], wq["scale"])["y"]
    assert bool(torch.isnan(z[rows]).all()) and torch.equal(z[~rows], y[~rows])
    h = tfla.gated_q8_fwd(bad_q["q"], bad_q["scale"], wq["q"], wq["scale"], wq["q"], wq["scale"])["hq"]
    k = tfla.gated_q8_fwd(good_q["q"], good_q["scale"], wq["q"], wq["scale"], wq["q"], wq["scale"])["hq"]
    assert bool(torch.isnan(h[rows].float()).all()) and torch.equal(h[~rows].view(torch.uint8), k[~rows].view(torch.uint8))
    n, m = tfla.norm_q8_fwd(bad), tfla.norm_q8_fwd(x)
    assert bool(torch.isnan(n["q"][1].float()).all()) and torch.equal(n["q"][~rows].view(torch.uint8), m["q"][~rows].view(torch.uint8))
    d = dy.clone()
    d[rows] = float("nan")
    o, p = (tfla.linear_q8_bwd(x, wq["qt"], wq["scale_t"], t, want_dw=False)["dx"] for t in (d, dy))
    assert bool(torch.isnan(o[rows]).all()) and torch.equal(o[~rows], p[~rows])
    # a scale of NaN
    s = good_q["scale"].view(torch.uint8).clone()
    s[0, 1] = 255
    z = tfla.linear_q8_fwd(good_q["q"], s.view(torch.float8_e8m0fnu), wq["q"], wq["scale"])["y"]
    rows[M - 1] = False
    assert bool(torch.isnan(z[rows]).all()) and torch.equal(z[~rows], y[~rows])


def test_small_and_large_scales(tfla):
    """groups next to the smallest and the largest exponents multiply as their powers of two say"""
    print("scales", flush=True)
    gen = generator(9)
    for M in (2, 70):
        x, w = ref.small_codes(gen, M, 256, 1), ref.small_codes(gen, 72, 256, 128)
        for e, f in ((0, 254), (247, 20), (1, 250), (100, 130)):
            xs, ws = torch.full_like(x[1].view(torch.uint8), e), torch.full_like(w[1].view(torch.uint8), f)
            y = tfla.linear_q8_fwd(x[0], xs.view(ref.E8M0), w[0], ws.view(ref.E8M0))["y"]
            z = (x[0].to(F64) @ w[0].to(F64).t()) * 2.0 ** (e + f - 254)
            assert torch.equal(y, z.float().to(BF16)), (M, e, f)


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("residual_block_8bit", os.path.join(ROOT, "examples", "residual_block_8bit.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_the_example_runs(example):
    print("example", flush=True)
    losses, worst = example.run(tokens=96, heads=2, dqk=64, dhv=64, steps=3)
    assert len(losses) == 3 and all(v == v for v in losses) and worst == worst


def test_the_examples_gradients_are_those_of_its_steps(example, tfla):
    """odd lengths; the feed-forward half's gradients by the same calls' 64-bit forms from what the forward pass left"""
    print("example gradients", flush=True)
    b = example.Block8(3, 64, 64)
    gen = generator(2)
    x, d = normal(gen, 1, 77, b.D), normal(gen, 1, 77, b.D)
    y, saved = b.forward(x)
    dx, g = b.backward(saved, d)
    assert y.shape == x.shape and dx.shape == x.shape
    assert set(g) == set(b.w) | set(b.v) and all(g[k].shape == (b.w | b.v)[k].shape and bool(torch.isfinite(g[k]).all()) for k in g)
    n2, h = saved[-2], saved[-1]
    (dh, edh), dws, _ = ref.back([d[0].to(F64)], [torch.zeros_like(d[0], dtype=F64)], h["h"], [ref.stands(*b._fwd("down"))])
    within("down", g["down"], *dws[0])
    down = tfla.linear_q8_bwd(h["h"], *b._bwd("down"), d[0])["dx"]
    within("dh", down, dh, edh)
    dz, ez = ref.gradients("silu", down, h["a"], h["u"])
    _, dws, _ = ref.back(dz, ez, n2["y"], [ref.stands(*b._fwd(k)) for k in ("gate", "up")])
    within("gate", g["gate"], *dws[0])
    within("up", g["up"], *dws[1])
