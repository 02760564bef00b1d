"""A residual block around the mLSTM cell on the framework's entry points: training steps, then generation token by token.

    pre-norm -> projections to q, k, v, the gates and the output gate -> cell with NORM and output gate -> projection back, plus
    the residual; pre-norm -> gated projection pair -> projection back, plus the residual.

Every matrix product, norm and cell runs in the library (linear_*, gated_*, norm_*, mlstm_layer_*); torch holds the memory, moves
heads next to each other and back, and does the optimizer's arithmetic.  The prompt is processed twice, as a whole and token by
token, and both have to agree.

    python examples/residual_block.py [--tokens 512] [--heads 4] [--dqk 64] [--dhv 128] [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2503_14376_amd as tfla  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


class Block:
    """Weights of one block and its passes.  heads * dhv is the model's width D; the feed-forward half is 8/3 as wide."""

    def __init__(self, heads, dqk, dhv, chunk=64, seed=0):
        self.h, self.dqk, self.dhv, self.chunk = heads, dqk, dhv, chunk
        D = self.D = heads * dhv
        F = self.F = (8 * D // 3 + 63) // 64 * 64
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n, k):
            return (torch.randn((n, k), generator=gen, device="cuda") * k ** -0.5).to(BF16)

        # one matrix for everything that reads the normed input: q, k, v, output gate, input and forget gates
        self.sizes = [heads * dqk, heads * dqk, D, D, heads, heads]
        self.w = {"in": weight(sum(self.sizes), D), "out": weight(D, D), "gate": weight(F, D), "up": weight(F, D), "down": weight(D, F)}
        bias = torch.zeros(sum(self.sizes), device="cuda")
        bias[-heads:] = 3.0                                           # forget gates start open
        self.v = {"b_in": bias, "g1": torch.ones(D, device="cuda"), "g2": torch.ones(D, device="cuda"),
                  "gh": torch.ones((heads, dhv), device="cuda")}

    def _split(self, p, B, T):
        """columns of the input projection -> per-head tensors (B, heads, T, width)"""
        parts = p.view(B, T, -1).split(self.sizes, dim=-1)
        heads = [t.reshape(B, T, self.h, -1).transpose(1, 2).contiguous() for t in parts[:4]]
        return heads + [t.transpose(1, 2).float().contiguous() for t in parts[4:]]

    def forward(self, x):
        """x: (B, T, D).  Returns the block's output and what backward needs."""
        B, T, D = x.shape
        w, v, x = self.w, self.v, x.reshape(B * T, D)
        n1 = tfla.norm_fwd(x, v["g1"])
        p = tfla.linear_fwd(n1["y"], w["in"], v["b_in"])["y"]
        q, k, u, o, i, f = self._split(p, B, T)
        c = tfla.mlstm_layer_fwd(q, k, u, i, f, o_pre=o, gamma=v["gh"], chunk=self.chunk, gate_softcap=15.0)
        y = c["Y"].transpose(1, 2).reshape(B * T, D)
        r = tfla.linear_fwd(y, w["out"], residual=x)["y"]
        n2 = tfla.norm_fwd(r, v["g2"])
        g = tfla.gated_fwd(n2["y"], w["gate"], w["up"], keep_pre=True)
        out = tfla.linear_fwd(g["h"], w["down"], residual=r)["y"]
        return out.view(B, T, D), (x, n1, q, k, u, o, i, f, c, y, r, n2, g)

    def backward(self, saved, d_out):
        """gradients of the weights and of the block's input"""
        x, n1, q, k, u, o, i, f, c, y, r, n2, g = saved
        B, T, D = d_out.shape
        w, v, d = self.w, self.v, d_out.reshape(B * T, D)
        down = tfla.linear_bwd(g["h"], w["down"], d)
        pair = tfla.gated_bwd(n2["y"], w["gate"], w["up"], g["a"], g["u"], down["dx"])
        nb2 = tfla.norm_bwd(r, pair["dx"], n2["rstd"], gamma=v["g2"], d_residual=d)
        out = tfla.linear_bwd(y, w["out"], nb2["dx"])
        dY = out["dx"].view(B, T, self.h, self.dhv).transpose(1, 2).contiguous()
        cb = tfla.mlstm_layer_bwd(q, k, u, i, f, c["H"], dY, o_pre=o, gamma=v["gh"], n_out=c["n_out"], m_out=c["m_out"],
                                  chunk=self.chunk, gate_softcap=15.0, want_dC0=False, fwd_workspace=c["workspace"])
        cols = [cb[n].transpose(1, 2).reshape(B * T, -1) for n in ("dq", "dk", "dv", "do_pre")]
        cols += [cb[n].transpose(1, 2).reshape(B * T, -1).to(BF16) for n in ("d_i_pre", "d_f_pre")]
        p = tfla.linear_bwd(n1["y"], w["in"], torch.cat(cols, dim=1), want_db=True)
        nb1 = tfla.norm_bwd(x, p["dx"], n1["rstd"], gamma=v["g1"], d_residual=nb2["dx"])
        grads = {"in": p["dw"], "out": out["dw"], "gate": pair["dw_gate"], "up": pair["dw_up"], "down": down["dw"], "b_in": p["db"],
                 "g1": nb1["dgamma"], "g2": nb2["dgamma"], "gh": cb["dgamma"]}
        return nb1["dx"].view(B, T, D), grads

    def step(self, x, state):
        """one token per sequence, x: (B, D); state: dict of C, n, m, replaced"""
        w, v, B = self.w, self.v, x.shape[0]
        n1 = tfla.norm_fwd(x, v["g1"])["y"]
        p = tfla.linear_fwd(n1, w["in"], v["b_in"])["y"]
        q, k, u, o, i, f = (t[:, :, 0].contiguous() for t in self._split(p, B, 1))
        s = tfla.mlstm_layer_step(q, k, u, i, f, state["C"], state["n"], state["m"], o_pre=o, gamma=v["gh"], gate_softcap=15.0)
        state.update(C=s["C"], n=s["n"], m=s["m"])
        r = tfla.linear_fwd(s["y"].reshape(B, self.D), w["out"], residual=x)["y"]
        h = tfla.gated_fwd(tfla.norm_fwd(r, v["g2"])["y"], w["gate"], w["up"])["h"]
        return tfla.linear_fwd(h, w["down"], residual=r)["y"]

    def empty_state(self, B):
        return {"C": torch.zeros((B, self.h, self.dqk, self.dhv), device="cuda"), "n": torch.zeros((B, self.h, self.dqk), device="cuda"),
                "m": torch.zeros((B, self.h), device="cuda")}


def run(tokens=512, heads=4, dqk=64, dhv=128, steps=20, batch=2, rate=0.02):
    """Trains a block to map a sequence onto another one and generates the prompt's outputs token by token.  Returns the losses
    and the largest difference between the two ways through the trained block, relative to the outputs' size."""
    block = Block(heads, dqk, dhv)
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
