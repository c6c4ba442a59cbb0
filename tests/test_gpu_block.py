"""The example's step of a gated feed-forward block (examples/finetune_block.py): joins with norms on both sides, gated
feed-forward, adapters, loss, their gradients and the step over all trained tensors together, against the same block in float64
(torch autograd on the CPU, frames from the oracle).

Tolerances: as for the library's other bf16 chains, 2e-2 normwise: the activations pass about a dozen roundings to bf16 (unit
roundoff 2^-8, mean error about 2^-9.5 each) between the loss and each gradient, 12^0.5 2^-9.5 = 0.5% where they are independent, and
a gradient of differences of those, as the norms' and the gate's are, some times that.  fp32: 1e-4."""
import importlib.util
import math
import os

import numpy as np
import pytest

from oracle import optim_oracle as OO
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
    spec = importlib.util.spec_from_file_location("finetune_block", os.path.join(ROOT, "examples", "finetune_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _block(example, dtype, width=256, hidden=512, vocab=300, T=70, nnz=900, rho=16, states="f32"):
    block = example.Block(width, hidden, vocab, T, nnz, rho=rho, alpha=60.0, seed=5, dtype=dtype, states=states)
    g = inputs.rng(6)
    for k, v in block.params.items():
        if k.startswith("C_"):
            plan = block.down if k == "C_d" else block.up
            v.copy_(torch.from_numpy(plan.to_plan(inputs.gaussian(g, (nnz,), std=0.05))))
        else:
            v.add_(torch.from_numpy(inputs.gaussian(g, (width,), std=0.1)).cuda())
    x, b = (torch.from_numpy(inputs.gaussian(g, (T, width), dtype="bf16")).to("cuda", dtype) for _ in range(2))
    target = torch.from_numpy(g.integers(0, vocab, T)).cuda()
    target[::7] = -100
    return block, x, b, target


def _float64(block, x, b, target, rho):
    f = torch.float64
    width, hidden = block.Wd.shape
    P = {d: torch.from_numpy(np.asarray(oracle_frame(d // rho, rho, d).toarray())) for d in (width, hidden)}
    q = {k: torch.from_numpy(to_np(v)).to(f).requires_grad_() for k, v in block.params.items()}
    x, b = (torch.from_numpy(to_np(t)).to(f).requires_grad_() for t in (x, b))
    Wg, Wu, Wd, head = (torch.from_numpy(to_np(t)).to(f) for t in (block.Wg, block.Wu, block.Wd, block.head))

    def adapter(v, name, plan, support, n, m):
        slot = torch.from_numpy(np.nonzero(plan.order >= 0)[0])
        user = torch.from_numpy(plan.order[plan.order >= 0])
        rows, cols = (torch.from_numpy(a.astype(np.int64)) for a in support)
        C = torch.zeros((m, n), dtype=f).index_put((rows[user], cols[user]), q[name][slot])
        return block.scale * (v @ P[n] @ C.t() @ P[m].t())

    def norm(v, name):
        return torch.nn.functional.rms_norm(v, (width,), q[name], 1e-5)

    x1 = x + norm(b, "norm_a")
    h1 = norm(x1, "norm_b")
    g = h1 @ Wg.t() + adapter(h1, "C_g", block.up, block.supports["up"], width, hidden)
    u = h1 @ Wu.t() + adapter(h1, "C_u", block.up, block.supports["up"], width, hidden)
    h = torch.nn.functional.silu(g) * u
    y = h @ Wd.t() + adapter(h, "C_d", block.down, block.supports["down"], hidden, width)
    h2 = norm(x1 + q["gate"] * norm(y, "norm_c"), "norm_d")
    t = target.cpu()
    loss = torch.nn.functional.cross_entropy(h2 @ head.t(), torch.where(t >= 0, t, -100), ignore_index=-100)
    loss.backward()
    return loss.item(), {k: v.grad.numpy() for k, v in q.items()}, x.grad.numpy(), b.grad.numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_step_matches_float64(example, dtype):
    block, x, b, target = _block(example, dtype)
    loss, share, grads, dx, db = block.gradients(x, b, target)
    torch.cuda.synchronize()
    want, ref, rx, rb = _float64(block, x, b, target, 16)
    tol = 2e-2 if dtype is torch.bfloat16 else 1e-4
    share = share.item()
    assert abs(loss.item() - want) <= tol * abs(want)
    for k in ref:
        assert rel(to_np(grads[k]) * share, ref[k]) <= tol, (k, rel(to_np(grads[k]) * share, ref[k]))
    assert rel(to_np(dx) * share, rx) <= tol and rel(to_np(db) * share, rb) <= tol


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_the_step_is_adamw_on_the_mean_gradient(example, states):
    """One whole step against the optimizer oracle on the gradients that the block gives: the decay of the coefficients alone, the
    mean's factor from the device, the first step's size."""
    block, x, b, target = _block(example, torch.bfloat16, states=states)
    _, share, grads, _, _ = block.gradients(x, b, target)
    before = {k: to_np(v) for k, v in block.params.items()}
    grads = {k: to_np(v) * share.item() for k, v in grads.items()}
    loss = block.step(x, b, target, 0.01)
    torch.cuda.synchronize()
    assert math.isfinite(loss.item())
    for k, v in block.params.items():
        zero = np.zeros_like(before[k])
        want, _, _ = OO.adamw_step(before[k], grads[k], zero, zero, 1, 0.01, weight_decay=0.01 if k.startswith("C_") else 0.0)
        # the first step is lr times the gradient's sign, whatever its size (eps 1e-8 below 1e-3 of it left out)
        sure = (np.abs(grads[k]) > 1e-5) | (grads[k] == 0)
        assert np.all(np.abs(to_np(v) - want)[sure] <= 1e-5 * (np.abs(before[k]) + 0.01)[sure]), k
        if k.startswith("C_"):
            pad = (block.down if k == "C_d" else block.up).order < 0
            assert not to_np(v)[pad].any()


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_example_runs(example, states):
    block = example.Block(256, 512, 1000, 128, 4000, rho=32, states=states)
    feed = example.batches(block, 128, 1)
    losses = [block.step(*next(feed), 0.01).item() for _ in range(5)]
    assert all(math.isfinite(v) for v in losses)


def test_whole_step_captured_and_replayed(example):
    """Gradients of the whole block and the optimizer's step captured once: every replay with other inputs equals an eager step from
    the same parameters; eager work of the same block runs between the replays."""
    block, x, b, target = _block(example, torch.bfloat16, states="8bit")
    twin, *_ = _block(example, torch.bfloat16, states="8bit")
    lr, number = torch.ones(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(bl):
        _, share, grads, _, _ = bl.gradients(x, b, target)
        bl.optimizer.step([grads[k] for k in bl.params], 0.01, 1, lr_dev=lr, grad_scale_dev=share, step_dev=number)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        twin.gradients(x, b, target)          # loads the kernels
        lr.zero_()
        step(block)                           # a step of no length, and moments cleared: the start again
        lr.fill_(1.0)
        s = block.optimizer
        for t in (s.m_all, s.v_all, s.m_exp_all, s.v_exp_all):
            t.zero_()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(block)
    for i in range(3):
        g = inputs.rng(40 + i)
        for t in (x, b):
            t.copy_(torch.from_numpy(inputs.gaussian(g, tuple(t.shape), dtype="bf16")).to("cuda", torch.bfloat16))
        number.fill_(i)
        lr.fill_(1.0 / (i + 1))
        graph.replay()
        step(twin)
        torch.cuda.synchronize()
        for k in block.params:
            assert torch.equal(block.params[k], twin.params[k]), (i, k)
        assert all(torch.equal(a, c) for a, c in zip(block.optimizer.read(), twin.optimizer.read()))
