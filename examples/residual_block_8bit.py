"""The residual block of examples/residual_block.py with its projections in 8 bits: training steps, then generation token by token.

    norm in 8 bits -> q, k, v and the output gate in 8 bits, the cell's gates in bf16 -> cell with NORM and output gate -> projection back in
    8 bits, plus the residual; norm in 8 bits -> gated pair, whose result leaves in 8 bits -> projection back, plus the residual.

Weights are quantised after every update, as they are (for the forward pass) and transposed (for the backward pass); the cell, the
gates' projection (its sums go through exponentials) and the residual stream stay as they were.

    python examples/residual_block_8bit.py [--tokens 512] [--heads 4] [--dqk 64] [--dhv 128] [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2503_14376_amd as tfla  # noqa: E402
from examples import residual_block  # noqa: E402

BF16 = torch.bfloat16


class Block8(residual_block.Block):
    def __init__(self, heads, dqk, dhv, chunk=64, seed=0):
        super().__init__(heads, dqk, dhv, chunk, seed)
        wide = sum(self.sizes[:4])
        self.w["gates"], self.v["b_gates"] = self.w["in"][wide:].contiguous(), self.v.pop("b_in")[wide:].contiguous()
        self.w["in"] = self.w["in"][:wide].contiguous()
        self.quantise()

    def quantise(self):
        """weights in 8 bits, plain and transposed: after every update"""
        self.q = {k: tfla.q8_quant(self.w[k], rows=128, want_t=True) for k in ("in", "out", "gate", "up", "down")}

    def _fwd(self, k):
        return self.q[k]["q"], self.q[k]["scale"]

    def _bwd(self, k):
        return self.q[k]["qt"], self.q[k]["scale_t"]

    def _quantised(self, x):
        o = tfla.q8_quant(x)
        return o["q"], o["scale"]

    def _project(self, n1):
        """a normed input in 8 bits and in bf16 -> columns of q, k, v, output gate, input and forget gates"""
        wide = tfla.linear_q8_fwd(n1["q"], n1["scale"], *self._fwd("in"))["y"]
        return torch.cat([wide, tfla.linear_fwd(n1["y"], self.w["gates"], self.v["b_gates"])["y"]], dim=1)

    def forward(self, x):
        B, T, D = x.shape
        v, x = self.v, x.reshape(B * T, D)
        n1 = tfla.norm_q8_fwd(x, v["g1"], keep_y=True)
        q, k, u, o, i, f = self._split(self._project(n1), B, T)
        c = tfla.mlstm_layer_fwd(q, k, u, i, f, o_pre=o, gamma=v["gh"], chunk=self.chunk, gate_softcap=15.0)
        y = c["Y"].transpose(1, 2).reshape(B * T, D)
        # the projection back and the residual's addition: the norm adds them up and goes on with the sum
        n2 = tfla.norm_q8_fwd(tfla.linear_q8_fwd(*self._quantised(y), *self._fwd("out"))["y"], v["g2"], residual=x, keep_y=True)
        g = tfla.gated_q8_fwd(n2["q"], n2["scale"], *self._fwd("gate"), *self._fwd("up"), keep_pre=True)
        out = tfla.linear_q8_fwd(g["hq"], g["h_scale"], *self._fwd("down"), residual=n2["sum"])["y"]
        return out.view(B, T, D), (x, n1, q, k, u, o, i, f, c, y, n2, g)

    def backward(self, saved, d_out):
        x, n1, q, k, u, o, i, f, c, y, n2, g = saved
        B, T, D = d_out.shape
        v, d = self.v, d_out.reshape(B * T, D)
        down = tfla.linear_q8_bwd(g["h"], *self._bwd("down"), d)
        pair = tfla.gated_q8_bwd(n2["y"], *self._bwd("gate"), *self._bwd("up"), g["a"], g["u"], down["dx"])
        nb2 = tfla.norm_bwd(n2["sum"], pair["dx"], n2["rstd"], gamma=v["g2"], d_residual=d)
        out = tfla.linear_q8_bwd(y, *self._bwd("out"), nb2["dx"])
        dY = out["dx"].view(B, T, self.h, self.dhv).transpose(1, 2).contiguous()
        cb = tfla.mlstm_layer_bwd(q, k, u, i, f, c["H"], dY, o_pre=o, gamma=v["gh"], n_out=c["n_out"], m_out=c["m_out"],
                                  chunk=self.chunk, gate_softcap=15.0, want_dC0=False, fwd_workspace=c["workspace"])
        wide = torch.cat([cb[n].transpose(1, 2).reshape(B * T, -1) for n in ("dq", "dk", "dv", "do_pre")], dim=1)
        narrow = torch.cat([cb[n].transpose(1, 2).reshape(B * T, -1).to(BF16) for n in ("d_i_pre", "d_f_pre")], dim=1)
        p = tfla.linear_q8_bwd(n1["y"], *self._bwd("in"), wide)
        pg = tfla.linear_bwd(n1["y"], self.w["gates"], narrow, want_db=True)
        nb1 = tfla.norm_bwd(x, p["dx"] + pg["dx"], n1["rstd"], gamma=v["g1"], d_residual=nb2["dx"])
        grads = {"in": p["dw"], "gates": pg["dw"], "b_gates": pg["db"], "out": out["dw"], "gate": pair["dw_gate"], "up": pair["dw_up"],
                 "down": down["dw"], "g1": nb1["dgamma"], "g2": nb2["dgamma"], "gh": cb["dgamma"]}
        return nb1["dx"].view(B, T, D), grads

    def step(self, x, state):
        v, B = self.v, x.shape[0]
        n1 = tfla.norm_q8_fwd(x, v["g1"], keep_y=True)
        q, k, u, o, i, f = (t[:, :, 0].contiguous() for t in self._split(self._project(n1), B, 1))
        s = tfla.mlstm_layer_step(q, k, u, i, f, state["C"], state["n"], state["m"], o_pre=o, gamma=v["gh"], gate_softcap=15.0)
        state.update(C=s["C"], n=s["n"], m=s["m"])
        y = tfla.linear_q8_fwd(*self._quantised(s["y"].reshape(B, self.D)), *self._fwd("out"))["y"]
        n2 = tfla.norm_q8_fwd(y, v["g2"], residual=x)
        g = tfla.gated_q8_fwd(n2["q"], n2["scale"], *self._fwd("gate"), *self._fwd("up"))
        return tfla.linear_q8_fwd(g["hq"], g["h_scale"], *self._fwd("down"), residual=n2["sum"])["y"]


def run(tokens=512, heads=4, dqk=64, dhv=128, steps=20, batch=2, rate=0.02):
    """Trains a block to map a sequence onto another one and generates the prompt's outputs token by token.  Returns the losses and the
    largest difference between the two ways through the trained block, relative to the outputs' size."""
    block = Block8(heads, dqk, dhv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((batch, tokens, block.D), generator=gen, device="cuda").to(BF16)
    goal = x.float().roll(1, dims=1)                # every token's output is to be the token before it
    goal[:, 0] = 0
    master = {k: t.float() for k, t in {**block.w, **block.v}.items()}
    losses = []
    for _ in range(steps):
        out, saved = block.forward(x)
        diff = out.float() - goal
        losses.append(float((diff * diff).mean()))
        _, grads = block.backward(saved, (diff * (2.0 / diff.numel()) * 1024.0).to(BF16))
        for k, g in grads.items():                  # normalised gradient steps on fp32 copies
            g = g.float()
            master[k] -= rate * g / (g.norm() / g.numel() ** 0.5 + 1e-12) * master[k].norm() / master[k].numel() ** 0.5
            (block.w if k in block.w else block.v)[k].copy_(master[k])
        block.quantise()
    whole, _ = block.forward(x)
    state, worst = block.empty_state(batch), 0.0
    for t in range(min(tokens, 64)):
        y = block.step(x[:, t].contiguous(), state)
        worst = max(worst, float((y.float() - whole[:, t].float()).abs().max()))
    return losses, worst / float(whole.float().abs().max())


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("tokens", 512), ("heads", 4), ("dqk", 64), ("dhv", 128), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    losses, worst = run(**vars(ap.parse_args()))
    print("loss %.4f -> %.4f over %d steps" % (losses[0], losses[-1], len(losses)))
    print("token by token against the whole prompt: largest difference %.2e of the largest output" % worst)


if __name__ == "__main__":
    main()
