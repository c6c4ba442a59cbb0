"""A fine-tuning step around one adapted projection, with the package's operators end to end.

    python examples/finetune_step.py [--steps 40] [--tokens 512] [--width 1024] [--vocab 5000]

The model is one pre-norm residual layer and a frozen head, as a transformer's last block is:

    h1 = norm(x)                                     layer norm, weight and bias trained
    y  = h1 W0^T + s P_out C P_in^T dropout(h1)      frozen projection, FrameFT adapter with input dropout
    x2 = x + dropout(y)
    loss = cross entropy of norm(x2) Wh^T            frozen head, logits never kept

Trained are C, and weight and bias of both norms, with AdamW.  Nothing that the backward pass could make
again is kept: no dropout mask, no normalised activations beyond those the projections read, no logits.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_26430_amd as ff  # noqa: E402
from paper_2608_26430_amd import inputs  # noqa: E402


class Layer:
    """The layer's frozen weights, its trained vectors with their AdamW state, and a step's workspaces."""

    def __init__(self, width, vocab, tokens, nnz, rho=64, p=0.1, alpha=20.0, seed=0, dtype=torch.bfloat16, device="cuda"):
        g = inputs.rng(seed)
        frame = ff.framegen(width, width // rho, rho)
        rows, cols = inputs.support(g, width, width, nnz)
        self.plan = ff.plan_create(frame, frame, rows, cols, max_tokens=tokens)
        self.p, self.seed, self.scale = p, seed, alpha / width

        def weight(m, n, std):
            return torch.from_numpy(inputs.gaussian(g, (m, n), std=std)).to(device, dtype)

        self.W0, self.head = weight(width, width, 1 / math.sqrt(width)), weight(vocab, width, 1 / math.sqrt(width))
        f32 = dict(dtype=torch.float32, device=device)
        self.params = {"C": torch.zeros(self.plan.coef_slots, **f32)}
        for name in ("norm1", "norm2"):
            self.params[name + ".weight"] = torch.ones(width, **f32)
            self.params[name + ".bias"] = torch.zeros(width, **f32)
        self.state = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in self.params.items()}
        self.ws_norm = ff.layernorm_workspace(tokens, width, device)
        self.ws_loss = ff.xent_workspace(tokens, width, vocab, dtype, want_dh=True, device=device)
        self.steps = 0

    def gradients(self, x, target, draw):
        """(mean loss over the tokens that have a target, gradients by name).  `draw` numbers the step's dropout masks."""
        q, p, seed = self.params, self.p, self.seed
        h1, m1, r1 = ff.layernorm_fwd(x, q["norm1.weight"], q["norm1.bias"])
        d = ff.dropout(h1, p, seed, 2 * draw)
        y = torch.mm(h1, self.W0.t())
        ff.adapter_fwd(self.plan, d, q["C"], self.scale, Y=y, beta=1.0)
        x2 = ff.dropout(y, p, seed, 2 * draw + 1, residual=x, Y=y)
        h2, m2, r2 = ff.layernorm_fwd(x2, q["norm2.weight"], q["norm2.bias"])
        counted = ((target >= 0) & (target < self.head.shape[0])).sum().clamp(min=1)
        share = 1.0 / counted.float()
        # Gradients of the tokens' sum: the mean's factor is known on the device only, and goes onto the fp32 results below.
        # As a weight of every token (dloss) it would be rounded to bf16 with the softmax, alike for all of them.
        loss, _, dh2, _ = ff.xent_step(h2, self.head, target, workspace=self.ws_loss)

        grads = {}
        dx2, grads["norm2.weight"], grads["norm2.bias"] = ff.layernorm_bwd(
            x2, dh2, q["norm2.weight"], m2, r2, workspace=self.ws_norm)
        dy = ff.dropout(dx2, p, seed, 2 * draw + 1)
        dd, grads["C"] = ff.adapter_bwd(self.plan, d, dy, q["C"], self.scale)
        dh1 = torch.mm(dy, self.W0)
        ff.dropout(dd, p, seed, 2 * draw, residual=dh1, Y=dh1)
        # (an earlier layer would also take dx = dx2 + the norm's dX, with beta_dx = 1)
        _, grads["norm1.weight"], grads["norm1.bias"] = ff.layernorm_bwd(
            x, dh1, q["norm1.weight"], m1, r1, want_dx=False, workspace=self.ws_norm)
        for g in grads.values():
            g.mul_(share)
        return loss.sum() * share, grads

    def step(self, x, target, lr):
        loss, grads = self.gradients(x, target, self.steps)
        self.steps += 1
        for name, w in self.params.items():
            m, v = self.state[name]
            ff.adamw_step(w, grads[name], m, v, lr, self.steps, weight_decay=0.01 if name == "C" else 0.0)
        return loss


def batches(layer, tokens, seed, skip=0.2):
    """Endless synthetic batches: activations N(0, 1), targets the head's answer to a fixed rotation of them; a share of
    the tokens (a prompt's) has none."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    width = layer.W0.shape[0]
    turn = torch.randn((width, width), generator=gen, device="cuda") / math.sqrt(width)
    while True:
        x = torch.randn((tokens, width), generator=gen, device="cuda").to(layer.W0.dtype)
        target = ((x.float() + x.float() @ turn) @ layer.head.float().t()).argmax(dim=1)
        target[torch.rand(tokens, generator=gen, device="cuda") < skip] = -100
        yield x, target


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--vocab", type=int, default=5000)
    ap.add_argument("--nnz", type=int, default=20_000)
    ap.add_argument("--lr", type=float, default=0.02)
    a = ap.parse_args()
    layer = Layer(a.width, a.vocab, a.tokens, a.nnz)
    feed = batches(layer, a.tokens, 1)
    for i in range(a.steps):
        x, target = next(feed)
        loss = layer.step(x, target, ff.lr_linear_warmup(i + 1, a.steps // 10, a.steps, a.lr))
        if i % 5 == 0 or i == a.steps - 1:
            print(f"step {i:3d}  loss {loss.item():.4f}", flush=True)


if __name__ == "__main__":
    main()
