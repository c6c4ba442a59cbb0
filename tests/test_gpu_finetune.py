"""The example's fine-tuning step (examples/finetune_step.py): layer norm, dropout, adapter, residual, loss and their
gradients together, against the same layer in float64 (torch autograd on the CPU, masks and frames from the oracles), and
training itself.

Tolerances: the activations pass about ten roundings to bf16 (unit roundoff 2^-8, mean error about 2^-9.5 each) between the
loss and each gradient; 2e-2 normwise, as for the library's other bf16 chains.  fp32: 1e-5 times the same ten stages, 1e-4."""
import importlib.util
import math
import os

import numpy as np
import pytest

from oracle import train_oracle as TO
from paper_2608_26430_amd import inputs
from tests.parity_util import oracle_frame, rel, to_np

torch = pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    spec = importlib.util.spec_from_file_location("finetune_step", os.path.join(ROOT, "examples", "finetune_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _float64(layer, x, target, draw, width, rho):
    """Loss and gradients of the layer by autograd in float64 on the CPU."""
    f = torch.float64
    P = torch.from_numpy(np.asarray(oracle_frame(width // rho, rho, width).toarray()))
    q = {k: torch.from_numpy(to_np(v)).to(f).requires_grad_() for k, v in layer.params.items()}
    order = layer.plan.order
    slot = torch.from_numpy(np.nonzero(order >= 0)[0])
    user = torch.from_numpy(order[order >= 0])
    rows, cols = (torch.from_numpy(a.astype(np.int64)) for a in layer.support)
    C = torch.zeros((width, width), dtype=f)
    C = C.index_put((rows[user], cols[user]), q["C"][slot])
    W0, head, x = (torch.from_numpy(to_np(t)).to(f) for t in (layer.W0, layer.head, x))
    T, keep = x.shape[0], 65536.0 / (65536 - TO.dropout_draws(layer.p))
    masks = [torch.from_numpy(TO.dropout_mask(T, width, layer.p, layer.seed, 2 * draw + i)).to(f) * keep for i in (0, 1)]

    def norm(v, name):
        return torch.nn.functional.layer_norm(v, (width,), q[name + ".weight"], q[name + ".bias"])

    h1 = norm(x, "norm1")
    y = h1 @ W0.t() + layer.scale * ((h1 * masks[0]) @ P @ C.t() @ P.t())
    z = norm(x + y * masks[1], "norm2") @ head.t()
    t = target.cpu()
    loss = torch.nn.functional.cross_entropy(z, torch.where(t >= 0, t, -100), ignore_index=-100)
    loss.backward()
    return loss.item(), {k: v.grad.numpy() for k, v in q.items()}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_step_matches_float64(example, dtype):
    width, vocab, T, nnz, rho = 256, 300, 70, 900, 16
    layer = example.Layer(width, vocab, T, nnz, rho=rho, p=0.2, alpha=60.0, seed=5, dtype=dtype)
    layer.support = inputs.support(inputs.rng(5), width, width, nnz)       # the draw that the layer made first
    g = inputs.rng(6)
    layer.params["C"].copy_(torch.from_numpy(layer.plan.to_plan(inputs.gaussian(g, (nnz,), std=0.05))))
    for k, v in layer.params.items():
        if k.endswith("weight"):
            v.add_(torch.from_numpy(inputs.gaussian(g, (width,), std=0.1)).cuda())
    x = torch.from_numpy(inputs.gaussian(g, (T, width), dtype="bf16")).to("cuda", dtype)
    target = torch.from_numpy(g.integers(0, vocab, T)).cuda()
    target[::7] = -100
    loss, grads = layer.gradients(x, target, draw=3)
    torch.cuda.synchronize()
    want, ref = _float64(layer, x, target, 3, width, rho)
    tol = 2e-2 if dtype is torch.bfloat16 else 1e-4
    assert abs(loss.item() - want) <= tol * abs(want)
    for k in ref:
        assert rel(to_np(grads[k]), ref[k]) <= tol, (k, rel(to_np(grads[k]), ref[k]))


def test_training_lowers_the_loss(example):
    layer = example.Layer(512, 1000, 256, 8000, rho=32)
    feed = example.batches(layer, 256, 1)
    losses = [layer.step(*next(feed), 0.02).item() for _ in range(30)]
    assert all(math.isfinite(v) for v in losses)
    assert np.mean(losses[-5:]) < np.mean(losses[:5]) - 0.05, losses


def test_gradients_are_the_differences(example):
    """Central differences of the fp32 layer's own loss (same masks) along a random direction of every trained tensor."""
    layer = example.Layer(256, 200, 64, 700, rho=16, p=0.1, alpha=60.0, seed=2, dtype=torch.float32)
    g = inputs.rng(3)
    layer.params["C"].copy_(torch.from_numpy(layer.plan.to_plan(inputs.gaussian(g, (700,), std=0.05))))
    x = torch.from_numpy(inputs.gaussian(g, (64, 256))).cuda()
    target = torch.from_numpy(g.integers(0, 200, 64)).cuda()
    _, grads = layer.gradients(x, target, draw=0)
    for k, v in layer.params.items():
        d = torch.from_numpy(inputs.gaussian(g, (v.numel(),))).cuda()
        if k == "C":
            d[torch.from_numpy(layer.plan.order < 0).cuda()] = 0
        d /= d.norm()
        keep, h = v.clone(), 0.05
        v.copy_(keep + h * d)
        up = layer.gradients(x, target, draw=0)[0].item()
        v.copy_(keep - h * d)
        down = layer.gradients(x, target, draw=0)[0].item()
        v.copy_(keep)
        got, want = float((grads[k] * d).sum()), (up - down) / (2 * h)
        # fp32 losses near 5: 2^-24 x 5 x about 30 operations over 2 h = 1e-4; third derivatives times h^2 / 6: 4e-4 of their size
        assert abs(got - want) <= 1e-4 + 5e-3 * abs(want) + 4e-4, (k, got, want)


def test_the_mean_over_tokens_is_not_rounded_alike(example):
    """Gradient at most targets is nearly minus one.  Over 510 counted tokens the mean's share of it lies just under the
    middle between two bf16 numbers (512 / 510 x 0.9995 = 1.0034 between 1 and 1.0078), so that rounding it would make all
    gradients 0.3% too small as a whole.  Rounded near one it is off by at most 2^-9 (0.9995 -> 1); what the other roundings
    leave is independent between elements and nearly cancels in this projection."""
    width, vocab, T, nnz, rho = 256, 1000, 512, 900, 16
    layer = example.Layer(width, vocab, T, nnz, rho=rho, p=0.1, seed=5)
    layer.support = inputs.support(inputs.rng(5), width, width, nnz)
    g = inputs.rng(8)
    x = torch.from_numpy(inputs.gaussian(g, (T, width), dtype="bf16")).to("cuda", torch.bfloat16)
    target = torch.from_numpy(g.integers(0, vocab, T)).cuda()
    target[:2] = -100
    _, grads = layer.gradients(x, target, draw=0)
    torch.cuda.synchronize()
    _, ref = _float64(layer, x, target, 0, width, rho)
    for k in ("norm2.weight", "norm2.bias"):
        share = float(np.sum((to_np(grads[k]) - ref[k]) * ref[k]) / np.sum(ref[k] ** 2))
        assert abs(share) <= 1.05 * 2.0 ** -9, (k, share)
