"""What examples/residual_block_8bit.py makes of the entry points: an update moves every weight against its gradient and is quantised anew, and a
token of the generation goes through the trained block's calls in the order of the formulas, each from what the one before it left."""
import importlib.util
import os

import pytest
import torch

from tests import q8_util as ref
from tests.block_util import F64, HALF, U, linear as linear64, norm as norm64, within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def tfla():
    import paper_2503_14376_amd as pkg
    pkg.load_library()
    return pkg


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("residual_block_8bit", os.path.join(ROOT, "examples", "residual_block_8bit.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def quantised_as_they_are(block):
    for k in ("in", "out", "gate", "up", "down"):
        ref.same_codes(block.q[k]["q"], block.q[k]["scale"], *ref.quant(block.w[k], 128), k)
        ref.same_codes(block.q[k]["qt"], block.q[k]["scale_t"], *ref.quant(block.w[k].t().contiguous(), 128), k + " transposed")


def test_an_update(example, tfla, monkeypatch):
    """one step of the example's training: w - rate g / rms(g) rms(w), and the codes of that"""
    print("update", flush=True)
    seen = []

    class Spy(example.Block8):
        def backward(self, saved, d_out):
            dx, grads = super().backward(saved, d_out)
            seen.append((self, {k: t.clone() for k, t in {**self.w, **self.v}.items()}, {k: g.clone() for k, g in grads.items()}))
            return dx, grads

    monkeypatch.setattr(example, "Block8", Spy)
    example.run(tokens=40, heads=2, dqk=64, dhv=64, steps=1, batch=1, rate=0.05)
    (block, before, grads), = seen
    after = {**block.w, **block.v}
    assert set(grads) == set(after)
    for k, g in grads.items():
        g, w = g.to(F64), before[k].to(F64)
        # (fp32: a sum of n squares, twice, and a handful of roundings of the step and of the result)
        move = 0.05 * g / (g.norm() / g.numel() ** 0.5 + 1e-12) * w.norm() / w.numel() ** 0.5
        assert bool((move != 0).any()), k
        within(k, after[k], w - move, (g.numel() + 8) * U * move.abs() + 2 * U * w.abs())
    quantised_as_they_are(block)


def test_a_token(example, tfla, monkeypatch):
    """step: every call's results by its 64-bit form, its inputs what the formulas say, after an update of the weights"""
    print("token", flush=True)
    B, block = 3, example.Block8(3, 64, 64)
    gen = torch.Generator(device="cuda").manual_seed(4)
    for k in block.w:
        block.w[k].mul_(1.5)
    for k in ("g1", "g2", "gh", "b_gates"):
        block.v[k].add_(torch.randn(block.v[k].shape, generator=gen, device="cuda") * 0.2)
    block.quantise()
    quantised_as_they_are(block)
    state, before = block.empty_state(B), None
    calls = []
    names = ("norm_q8_fwd", "linear_q8_fwd", "linear_fwd", "mlstm_layer_step", "q8_quant", "gated_q8_fwd")

    def spied(name, call):
        def run(*a, **kw):
            o = call(*a, **kw)
            calls.append((name, a, kw, o))
            return o
        return run
    for name in names:
        monkeypatch.setattr(tfla, name, spied(name, getattr(tfla, name)))
    for token in range(3):
        x = (torch.randn((B, block.D), generator=gen, device="cuda")).to(BF16)
        before = dict(state)
        calls.clear()
        y = block.step(x, state)
        n1, wide, gates, cell, again, back, n2, pair, down = calls
        assert [c[0] for c in calls] == ["norm_q8_fwd", "linear_q8_fwd", "linear_fwd", "mlstm_layer_step", "q8_quant", "linear_q8_fwd", "norm_q8_fwd",
                                         "gated_q8_fwd", "linear_q8_fwd"]
        stands = {k: ref.stands(*block._fwd(k)) for k in block.q}
        # the norm of x, with the values that the gates' projection takes
        assert n1[1][0] is x
        _, _, (v, ev) = norm64(x, block.v["g1"], None, False, 1e-6)
        within("n1", n1[3]["y"], v, ev)
        half = HALF[BF16]               # (the codes are those of y before its rounding)
        ref.coded("n1", n1[3]["q"], n1[3]["scale"], n1[3]["y"].to(F64), half * n1[3]["y"].to(F64).abs())
        # projections: q, k, v and the output gate from codes, the gates from bf16
        (v, ev), _ = ref.linear(ref.stands(n1[3]["q"], n1[3]["scale"]), stands["in"], None, None, "none")
        within("wide", wide[3]["y"], v, ev)
        (v, ev), _ = linear64(n1[3]["y"], block.w["gates"], block.v["b_gates"], None, "none")
        within("gates", gates[3]["y"], v, ev)
        # the cell on those columns, head by head, from the state that the token before left
        parts = torch.cat([wide[3]["y"], gates[3]["y"]], dim=1).split(block.sizes, dim=1)
        q, k, u, o, i, f = (t.reshape(B, block.h, -1) for t in parts)
        a, kw = cell[1], cell[2]
        for got, want in zip(a[:3], (q, k, u)):
            assert torch.equal(got, want)
        assert torch.equal(kw["o_pre"], o) and torch.equal(a[3], i[:, :, 0].float()) and torch.equal(a[4], f[:, :, 0].float())
        assert a[5] is before["C"] and a[6] is before["n"] and a[7] is before["m"] and torch.equal(kw["gamma"], block.v["gh"])
        assert all(state[s] is cell[3][s] for s in ("C", "n", "m"))
        # back, and the residual
        heads = cell[3]["y"].reshape(B, block.D)
        ref.same_codes(again[3]["q"], again[3]["scale"], *ref.quant(heads), "heads")
        (v, ev), _ = ref.linear(ref.stands(again[3]["q"], again[3]["scale"]), stands["out"], None, None, "none")
        within("back", back[3]["y"], v, ev)
        assert n2[1][0] is back[3]["y"] and n2[2]["residual"] is x
        total = back[3]["y"].to(F64) + x.to(F64)
        within("sum", n2[3]["sum"], total, U * total.abs())
        _, _, (v, ev) = norm64(total.float(), block.v["g2"], None, False, 1e-6)
        ref.coded("n2", n2[3]["q"], n2[3]["scale"], v, ev)
        # the feed-forward half
        _, _, (v, ev) = ref.gated(ref.stands(n2[3]["q"], n2[3]["scale"]), stands["gate"], stands["up"], None, None, "silu")
        ref.coded("h", pair[3]["hq"], pair[3]["h_scale"], v, ev)
        _, (v, ev) = ref.linear(ref.stands(pair[3]["hq"], pair[3]["h_scale"]), stands["down"], None, n2[3]["sum"], "none")
        within("y", y, v, ev)
