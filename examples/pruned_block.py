"""A feed-forward block whose hidden channels the projection prunes: trained, projected after every step, packed to
4 bits and asked token by token.

    python examples/pruned_block.py

The block is  r = x + scale * gate * norm(h Wd),  y = norm(r)  with  h = silu(z Wg) * (z Wu)  and  z = norm(x).  It learns a
teacher of the same form with few hidden channels; the l1,inf projection of Wg after every step leaves the channels that
matter and the mask that the block's products skip the others by.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2405_02086_amd import binding as mp  # noqa: E402


class PrunedBlock:
    """bf16 weights with fp32 masters; columns of Wg and Wu, rows of Wd are the hidden channels."""

    def __init__(self, n, m, generator, scale=0.5, kept=None):
        def weight(rows, cols):
            return torch.randn(rows, cols, generator=generator, device="cuda") / rows ** 0.5
        self.scale = scale
        self.master = {"Wg": weight(n, m), "Wu": weight(n, m), "Wd": weight(m, n), "w_in": torch.ones(n, device="cuda"),
                       "w_post": torch.ones(n, device="cuda"), "gate": torch.ones(n, device="cuda"),
                       "w_out": torch.ones(n, device="cuda")}
        if kept is not None:
            for name in ("Wg", "Wu"):
                self.master[name][:, kept:] = 0
        self.mask = torch.ones(m, dtype=torch.uint8, device="cuda")
        self.cast()

    def cast(self):
        self.w = {k: v.to(torch.bfloat16) for k, v in self.master.items()}

    def forward(self, x):
        w = self.w
        _, z = mp.block_norm(x, w_pre=w["w_in"])
        h = mp.gated_ff(z, w["Wg"], w["Wu"], mask=self.mask)
        b = h @ w["Wd"]
        r, y = mp.block_norm(x, b, w["w_post"], w["gate"], w["w_out"], scale=self.scale)
        return y, (x, z, h, b, r)

    def backward(self, dy, saved):
        """Gradients of the weights for the gradient dy of the result."""
        w = self.w
        x, z, h, b, r = saved
        _, db, dw_post, dgate, dw_out = mp.block_norm_backward(None, dy, r, b, w["w_post"], w["gate"], w["w_out"], scale=self.scale)
        dz, dWg, dWu = mp.gated_ff_backward(db @ w["Wd"].t(), z, w["Wg"], w["Wu"], mask=self.mask)
        _, _, _, _, dw_in = mp.block_norm_backward(None, dz, x, w_pre=w["w_in"])
        return {"Wg": dWg, "Wu": dWu, "Wd": h.t() @ db, "w_in": dw_in, "w_post": dw_post, "gate": dgate, "w_out": dw_out}

    def step(self, gradients, rate):
        for k, g in gradients.items():
            self.master[k].sub_(g.float(), alpha=rate)
        self.cast()

    def project(self, eta):
        """The l1,inf projection of Wg; pruned channels leave Wu as well."""
        mp.bilevel_proj_stored(self.w["Wg"], eta, "inf", X=self.w["Wg"], mask_out=self.mask)
        self.master["Wg"].copy_(self.w["Wg"])
        self.master["Wu"].mul_(self.mask)
        self.w["Wu"].mul_(self.mask)

    def packed(self, group=64):
        return {k: mp.w4_pack(self.w[k], group) for k in ("Wg", "Wu", "Wd")}

    def answer(self, x, packed):
        """The block on a few tokens with packed weights."""
        w = self.w
        _, z = mp.block_norm(x, w_pre=w["w_in"])
        h = mp.w4_gated_matvec(z, packed["Wg"], packed["Wu"])
        b = mp.w4_matvec(h, packed["Wd"])
        return mp.block_norm(x, b, w["w_post"], w["gate"], w["w_out"], scale=self.scale)[1]


def main(n=256, m=512, relevant=48, tokens=512, steps=60, rate=16.0, radius=0.03, seed=0):
    """Trains; returns what `python examples/pruned_block.py` prints."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    teacher = PrunedBlock(n, m, gen, kept=relevant)
    block = PrunedBlock(n, m, gen)
    eta = radius * float(block.master["Wg"].abs().amax(0).sum())
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, n, generator=gen, device="cuda").to(torch.bfloat16)
        target, _ = teacher.forward(x)
        y, saved = block.forward(x)
        off = y.float() - target.float()
        losses.append(float((off * off).mean()))
        block.step(block.backward((2 * off / tokens).to(torch.bfloat16), saved), rate / n)
        block.project(eta)
    packed = block.packed()
    x = torch.randn(1, n, generator=gen, device="cuda").to(torch.bfloat16)
    exact, short = block.forward(x)[0].float(), block.answer(x, packed).float()
    return {"first_loss": losses[0], "last_loss": losses[-1], "kept": int(block.mask.sum()), "channels": m,
            "four_bit_error": float((short - exact).norm() / exact.norm())}


if __name__ == "__main__":
    for key, value in main().items():
        print(key, value)
