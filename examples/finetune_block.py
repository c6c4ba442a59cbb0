"""A fine-tuning step of a gated feed-forward block with adapters on its three projections, with the package's operators end to end.

    python examples/finetune_block.py [--steps 40] [--tokens 512] [--width 512] [--hidden 1024] [--vocab 5000] [--states 8bit]

The model is the second half of a transformer's block with norms on both sides of it, and a frozen head:

    x1 = x + norm_a(b),  h1 = norm_b(x1)             b: what the block before has put out
    g  = h1 Wg^T + adapter_g(h1),  u = h1 Wu^T + adapter_u(h1),  h = silu(g) u
    y  = h Wd^T + adapter_d(h)
    x2 = x1 + gate norm_c(y),  h2 = norm_d(x2)       a learned gate for each channel
    loss = cross entropy of h2 Wh^T                  frozen head, logits never kept

Trained are the adapters' coefficients, the norms' weights and the gate, by one AdamW step over all of them, with moments in fp32 or
in 8 bits.  Between forward and backward are kept: the norms' inputs and statistics, h1, g, u and h.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_26430_amd as ff  # noqa: E402
from paper_2608_26430_amd import inputs  # noqa: E402

NORMS = ("norm_a", "norm_b", "norm_c", "norm_d")


class Block:
    """The block's frozen weights, what is trained of it, and a step's workspaces."""

    def __init__(self, width, hidden, vocab, tokens, nnz, rho=64, alpha=20.0, seed=0, dtype=torch.bfloat16, states="f32",
                 device="cuda"):
        g = inputs.rng(seed)
        f_n, f_h = ff.framegen(width, width // rho, rho), ff.framegen(hidden, hidden // rho, rho)
        self.supports = {"up": inputs.support(g, hidden, width, nnz), "down": inputs.support(g, width, hidden, nnz)}
        # the gate and up projections share a support, and with it a plan
        self.up = ff.plan_create(f_n, f_h, *self.supports["up"], max_tokens=tokens)
        self.down = ff.plan_create(f_h, f_n, *self.supports["down"], max_tokens=tokens)
        self.scale = alpha / math.sqrt(width * hidden)

        def weight(m, n):
            return torch.from_numpy(inputs.gaussian(g, (m, n), std=1 / math.sqrt(n))).to(device, dtype)

        self.Wgu, self.Wd, self.head = weight(2 * hidden, width), weight(width, hidden), weight(vocab, width)
        self.Wg, self.Wu = self.Wgu[:hidden], self.Wgu[hidden:]
        f32 = dict(dtype=torch.float32, device=device)
        self.params = {"C_g": torch.zeros(self.up.coef_slots, **f32), "C_u": torch.zeros(self.up.coef_slots, **f32),
                       "C_d": torch.zeros(self.down.coef_slots, **f32), "gate": torch.ones(width, **f32)}
        for name in NORMS:
            self.params[name] = torch.ones(width, **f32)
        self.optimizer = ff.AdamWSet(list(self.params.values()), states=states, seed=seed,
                                     weight_decay=[0.01 if k.startswith("C_") else 0.0 for k in self.params])
        self.ws_join = ff.resnorm_workspace(tokens, width, device=device)
        self.ws_glu = ff.glu_workspace(tokens, width, hidden, dtype, device=device)
        self.ws_loss = ff.xent_workspace(tokens, width, vocab, dtype, want_dh=True, device=device)
        self.steps = 0

    def gradients(self, x, b, target):
        """(mean loss over the tokens that have a target, its factor on the gradients (a device value), gradients of the tokens'
        sum by name, gradients of x and of b)."""
        q, s = self.params, self.scale
        join1 = dict(post="rms", post_weight=q["norm_a"], norm="rms", weight=q["norm_b"])
        join2 = dict(gate=q["gate"], post="rms", post_weight=q["norm_c"], norm="rms", weight=q["norm_d"])
        x1, h1, st1 = ff.resnorm_fwd(x, b, **join1)
        a_g, a_u = ff.adapter_fwd(self.up, h1, q["C_g"], s), ff.adapter_fwd(self.up, h1, q["C_u"], s)
        h, g, u = ff.glu_fwd(h1, self.Wg, self.Wu, "silu", a_g, a_u, save=True)
        y = torch.mm(h, self.Wd.t())
        ff.adapter_fwd(self.down, h, q["C_d"], s, Y=y, beta=1.0)
        _, h2, st2 = ff.resnorm_fwd(x1, y, **join2)
        counted = ((target >= 0) & (target < self.head.shape[0])).sum().clamp(min=1)
        loss, _, dh2, _ = ff.xent_step(h2, self.head, target, workspace=self.ws_loss)

        grads = {}
        # x2 goes nowhere but into the last norm: no gradient from the stream
        dx1, dy, grads["gate"], grads["norm_c"], _, grads["norm_d"], _ = ff.resnorm_bwd(
            x1, y, None, dh2, st2, workspace=self.ws_join, **join2)
        dh = torch.mm(dy, self.Wd)
        _, grads["C_d"] = ff.adapter_bwd(self.down, h, dy, q["C_d"], s, dX=dh, beta_dx=1.0)
        # dg and du take the place of g and u
        dg, du, dh1, _, _ = ff.glu_bwd(dh, h1, self.Wg, self.Wu, "silu", G=g, U=u, dG=g.view(x.dtype), dU=u.view(x.dtype),
                                      workspace=self.ws_glu)
        _, grads["C_g"] = ff.adapter_bwd(self.up, h1, dg, q["C_g"], s, dX=dh1, beta_dx=1.0)
        _, grads["C_u"] = ff.adapter_bwd(self.up, h1, du, q["C_u"], s, dX=dh1, beta_dx=1.0)
        dx, db, _, grads["norm_a"], _, grads["norm_b"], _ = ff.resnorm_bwd(
            x, b, dx1, dh1, st1, dR=dx1, workspace=self.ws_join, **join1)
        share = 1.0 / counted.float()
        return loss.sum() * share, share, grads, dx, db

    def step(self, x, b, target, lr):
        loss, share, grads, _, _ = self.gradients(x, b, target)
        self.steps += 1
        # the mean's factor is known on the device only
        self.optimizer.step([grads[k] for k in self.params], lr, self.steps, grad_scale_dev=share)
        return loss


def batches(block, tokens, seed, skip=0.2):
    """Endless synthetic batches: activations N(0, 1), targets the head's answer to a fixed mixture of both inputs; a share of
    the tokens (a prompt's) has none."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    width = block.Wd.shape[0]
    turn = torch.randn((width, width), generator=gen, device="cuda") / math.sqrt(width)
    while True:
        x, b = (torch.randn((tokens, width), generator=gen, device="cuda").to(block.Wd.dtype) for _ in range(2))
        target = ((x.float() + b.float() @ turn) @ block.head.float().t()).argmax(dim=1)
        target[torch.rand(tokens, generator=gen, device="cuda") < skip] = -100
        yield x, b, target


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--vocab", type=int, default=5000)
    ap.add_argument("--nnz", type=int, default=20_000)
    ap.add_argument("--lr", type=float, default=0.02)
    ap.add_argument("--states", choices=("f32", "8bit"), default="f32")
    a = ap.parse_args()
    block = Block(a.width, a.hidden, a.vocab, a.tokens, a.nnz, states=a.states)
    feed = batches(block, a.tokens, 1)
    for i in range(a.steps):
        x, b, target = next(feed)
        loss = block.step(x, b, target, ff.lr_linear_warmup(i + 1, a.steps // 10, a.steps, a.lr))
        if i % 5 == 0 or i == a.steps - 1:
            print(f"step {i:3d}  loss {loss.item():.4f}", flush=True)


if __name__ == "__main__":
    main()
