"""The head's loss on the sizes it is made for: the 256 x 256 tiles of every product and the walk of one workgroup over several
of them, pieces of tokens and of the vocabulary with a short last one, rows past one launch's second dimension.  Which tiles
and pieces a case runs is pinned on the CPU by test_loss_plans.py.

The reference is the formula in 64 bits on the device.  Bounds per element as in test_gpu_xent.py; besides, every row of dH and
dW is off by at most 2e-2 of its own norm (an element's bound is a worst case over all terms; a row's rounding errors are
independent, so that this finds a wrong piece of a row which the sums of absolute values would cover)."""
import numpy as np
import pytest

from tests.parity_util import TOL

torch = pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402

pytestmark = pytest.mark.gpu
V32 = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
LARGE, MEDIUM, SMALL, TINY = range(4)

# tokens, width, entries, type, dH, dW, what the plan has to be: tile of each product, products whose workgroups walk several
# tiles (more than 256 of the large one), pieces of the gradient (vocabulary or tokens), pieces of the forward by itself
CASES = [
    (2500, 2056, 33001, "bf16", True, True, dict(logits=LARGE, dh=LARGE, dw=LARGE, walks="logits dh dw", pieces=1, forwards=1)),
    (7500, 4104, 17001, "bf16", True, False, dict(logits=LARGE, dh=LARGE, walks="logits dh", split=1, pieces=1, forwards=1)),
    # the last piece of the vocabulary is shorter than the split of dH: some of its sums are of nothing
    (4200, 2056, 33003, "bf16", True, True, dict(logits=LARGE, dh=LARGE, dw=LARGE, walks="logits dh dw", pieces=2, forwards=1)),
    (9000, 520, 32003, "bf16", True, True, dict(logits=LARGE, pieces=3, forwards=2)),
    (5000, 264, 60001, "bf16", True, False, dict(logits=LARGE, dh=MEDIUM, walks="logits", pieces=3, forwards=2)),
    (2000, 264, 250_001, "bf16", False, False, dict(logits=LARGE, walks="logits", forwards=2)),
    (260, 8, 1_000_003, "bf16", False, False, dict(forwards=2)),
    (260, 8, 1_000_003, "f32", False, False, dict(logits=MEDIUM, forwards=2)),
    (40_000, 16, 20, "bf16", True, True, dict(pieces=1, forwards=1)),
    (40_000, 16, 20, "f32", True, True, dict(pieces=1, forwards=1)),
]


def _reference(H, W, target, dloss, scale, grads):
    """loss, lse, zabs and, with grads, (dH, sum |P| |W|), (dW, sum |P| |H|) in float64."""
    f64 = torch.float64
    T, V = H.shape[0], W.shape[0]
    Wd = W.to(f64)
    Wa = Wd.abs()
    loss, lse, zabs = (torch.zeros(T, dtype=f64, device=H.device) for _ in range(3))
    dH, dHa = (torch.zeros(H.shape, dtype=f64, device=H.device) for _ in range(2))
    dW, dWa = (torch.zeros(W.shape, dtype=f64, device=H.device) for _ in range(2))
    rows = max(1, min(T, (1 << 27) // V))
    for t in range(0, T, rows):
        s = slice(t, min(T, t + rows))
        h = H[s].to(f64)
        z = h @ Wd.t()
        lse[s] = torch.logsumexp(z, dim=1)
        zabs[s] = (h.abs() @ Wa.t()).amax(dim=1)
        live = (target[s] >= 0) & (target[s] < V)
        at = torch.where(live, target[s], 0)[:, None]
        loss[s] = torch.where(live, lse[s] - z.gather(1, at)[:, 0], 0.0)
        if not grads:
            continue
        P = torch.exp(z - lse[s][:, None]).scatter_(1, at, 0.0)
        P.scatter_(1, at, -P.sum(dim=1, keepdim=True))
        P *= (torch.where(live, dloss[s].to(f64), 0.0) * scale)[:, None]
        dH[s], dHa[s] = P @ Wd, P.abs() @ Wa
        dW += P.t() @ h
        dWa += P.abs().t() @ h.abs()
    return loss, lse, zabs, (dH, dHa), (dW, dWa)


@pytest.mark.parametrize("T,n,V,dtype,want_dh,want_dw,plan", CASES)
def test_large_calls_match_float64(T, n, V, dtype, want_dh, want_dw, plan):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    dev, dt, u = torch.device("cuda:0"), torch.bfloat16 if dtype == "bf16" else torch.float32, U[dtype]
    gen = torch.Generator(device=dev)
    gen.manual_seed(T + n + V)

    def randn(rows, std=1.0):
        """rows x n inside rows of n + 8, NaN beside them"""
        buf = torch.full((rows, n + 8), float("nan"), device=dev, dtype=dt)
        buf[:, :n] = torch.randn((rows, n), generator=gen, device=dev) * std
        return buf[:, :n], buf

    (H, _), (W, _) = randn(T), randn(V, 2.0 / np.sqrt(n))
    target = torch.randint(0, V, (T,), generator=gen, device=dev)
    target[torch.rand(T, generator=gen, device=dev) < 0.2] = -100
    dloss = torch.rand(T, generator=gen, device=dev) + 0.25
    grads, scale, beta = want_dh or want_dw, 0.3, 0.5
    loss64, lse64, zabs, *products = _reference(H, W, target, dloss, scale, grads)
    Ez = (n / 16 + 48) * 2 * V32 * zabs
    El = 2 * Ez + 16 * V32 * (1 + lse64.abs() + zabs) + (V / 64 + 64) * V32
    rp = 2 * float(Ez.max()) + 3 * u + 32 * V32 + 64 * V32 * 90

    def check_loss(loss, lse):
        assert bool(((loss - loss64).abs() <= 1.05 * El).all()) and bool(((lse - lse64).abs() <= 1.05 * El).all())
        assert bool((loss[target < 0] == 0).all())

    def check_grads(got, bufs, olds):
        for out, buf, old, (want, sums), terms in zip(got, bufs, olds, products, (V, T)):
            if out is None:
                continue
            total = want + beta * old
            bound = (rp + (terms / 16 + 48) * 2 * V32) * sums + u * total.abs() + 4 * V32 * old.abs()
            d = (out.double() - total).abs()
            assert bool((d <= 1.05 * bound + 1e-37).all()), float((d / (bound + 1e-37)).max())
            rows = torch.linalg.vector_norm(out.double() - beta * old - want, dim=1)
            # the old value's and the result's own rounding come on top of the row's errors
            floor = 2 * u * torch.linalg.vector_norm(total, dim=1)
            assert bool((rows <= TOL["bf16"] * torch.linalg.vector_norm(want, dim=1) + floor + 1e-37).all())
            assert bool(torch.isnan(buf[:, n:]).all())

    ws = ff.xent_workspace(T, n, V, dt, want_dh=want_dh, want_dw=want_dw, device=dev)
    ws.fill_(255)
    loss, lse = ff.xent_fwd(H, W, target, workspace=ws)
    check_loss(loss, lse)
    if not grads:
        return
    for step in (True, False):
        (dH, bh), (dW, bw) = randn(T), randn(V)
        olds = dH.double(), dW.double()
        out = dict(dH=dH if want_dh else None, dW=dW if want_dw else None, beta_dh=beta if want_dh else 0.0,
                   beta_dw=beta if want_dw else 0.0, want_dh=want_dh, want_dw=want_dw, workspace=ws)
        ws.fill_(255)
        if step:
            loss2, lse2, gh, gw = ff.xent_step(H, W, target, dloss=dloss, scale=scale, **out)
            check_loss(loss2, lse2)
        else:
            gh, gw = ff.xent_bwd(H, W, target, lse, loss=loss, dloss=dloss, scale=scale, **out)
        check_grads((gh, gw), (bh, bw), olds)
