"""Every instance of the join's kernels: each kind of norms, with and without a gate, at sizes that reach each number of pieces and
waves with and without a last piece that overlaps the one before (test_resnorm_plans.py asks which); the statistics against
bounds of their own.  References and bounds are those of test_gpu_resnorm.py."""
import numpy as np
import pytest

from paper_2608_26430_amd import inputs
from tests.parity_util import to_np
from tests.test_gpu_resnorm import (BLOCK, EPS, OUT, RES, U, V, _strided, bounds, case, check, close, device_args, reference, run)

torch = pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    return torch.device("cuda:0")


# rows longer and shorter than 512 where the choice asks; a multiple of every piece, and odd ones
SIZES = [(37, 200), (37, 203), (600, 509), (20, 500), (20, 504), (600, 1021), (600, 1016), (20, 1021), (20, 1016), (20, 1531), (600, 1531), (20, 1528), (20, 2045), (20, 2048),
         (20, 3001), (520, 3003), (20, 3000), (9, 5003), (9, 5000), (9, 8189), (9, 8192), (5, 9001), (5, 16392)]
# post, norm, biases: the six groups of instances of the backward
KINDS = [("rms", "rms", False), ("layer", "layer", True), ("none", "rms", False), ("none", "layer", True), ("rms", "none", True),
         ("none", "none", False)]


@pytest.mark.parametrize("T,n", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_kind_with_and_without_a_gate(dev, T, n, dtype):
    for i, (post, norm, bias) in enumerate(KINDS):
        for gate in (0, 1):
            c = case(T, n, dtype, post, norm, gate, 10 * T + n + i, bias=bias)
            X, Y, stats, grads, act, how = run(c, dtype, dev, post, norm)
            again = ff.resnorm_bwd(act["r"], act["b"], act["dx"], act["dy"], stats, **how)
            torch.cuda.synchronize()
            check(c, dtype, post, norm, X, Y, stats, grads)
            check_statistics(c, post, norm, stats)
            assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("T,n,ld,at", [(37, 1531, 1533, 1), (37, 3001, 3003, 1), (37, 5003, 5003, 3), (530, 1021, 1024, 1), (530, 1531, 1533, 1),
                                       (520, 3003, 3003, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_over_inputs_with_overlapping_last_pieces(dev, T, n, ld, at, dtype):
    """x over r, dr over dx, db over dy or b, where a row's last piece shares elements with another wave's; nothing else is written."""
    for post, norm, bias in KINDS:
        c = case(T, n, dtype, post, norm, 1, n + T, bias=bias)
        t = {k: _strided(c[k], dtype, dev, ld, at) for k in ("r", "b", "dx", "dy") if c[k] is not None}
        how = dict(post=post, norm=norm, res_scale=RES, block_scale=BLOCK, eps=EPS, **device_args(c, dtype, dev))
        r2, around = _strided(c["r"], dtype, dev, ld, at)
        X, Y, stats = ff.resnorm_fwd(r2, t["b"][0], X=r2, **how)
        over = t["dy"][0] if norm != "none" else t["b"][0]
        grads = ff.resnorm_bwd(t["r"][0], t["b"][0], t["dx"][0], t["dy"][0] if norm != "none" else None, stats, dR=t["dx"][0], dB=over, **how)
        torch.cuda.synchronize()
        o = reference(c, post, norm)
        B = bounds(o, c, post, norm, U[dtype])
        close(X, o["x"], B["x"], "x")
        if norm != "none":
            close(Y, o["y"], B["y"], "y")
        for k, g in zip(OUT, grads):
            if g is not None:
                close(g, o[k], B[k], k)
        for name, (_, buf) in list(t.items()) + [("x", (None, around))]:
            out = np.ones(buf.numel(), dtype=bool)
            out[(np.arange(T)[:, None] * ld + at + np.arange(n)[None, :]).ravel()] = False
            assert np.isnan(to_np(buf)[out]).all(), (name, post, norm)


def check_statistics(c, post, norm, stats):
    """Mean and 1 / deviation of b and of x.  Sums of fp32 values in fp32: at most 32 terms a thread and 10 levels (rows over 8192: below), 42 v of the absolute
    terms' sum, and v for the division: a mean is off by em = 43 v mean|x|, beside what the values are off by, mean e; the centred
    square's mean by 2 v + 42 v of itself and by the first order of the centred values' errors d = e + em + v |x - mean|, 2 mean(|x -
    mean| d), which is at most 2 sigma rms(d), and mean d^2; 1 / deviation by half of that relative and 3 v of the root, the sum
    with eps and the division."""
    o = reference(c, post, norm)
    got, n = to_np(stats).astype(np.float64), c["r"].shape[1]
    terms = 42 if n <= 8192 else 22 + -(-n // 1024)       # (rows of any width: 1024 threads, 6 levels and 16 waves)
    bound_x = bounds(o, c, post, norm, 0.0)["x"] if norm != "none" else None
    for kind, x, e, mean, rstd, at in ((post, np.asarray(c["b"], dtype=np.float64), 0.0, o["mp"], o["rp"], 0), (norm, o["x"], bound_x, o["m"], o["q"], 2)):
        if kind == "none":
            assert not got[:, at:at + 2].any()
            continue
        e = np.zeros_like(x) if at == 0 else e
        em = np.zeros_like(mean)
        if kind == "layer":
            em = (terms + 1) * V * np.abs(x).mean(axis=1, keepdims=True) + e.mean(axis=1, keepdims=True)
            assert (np.abs(got[:, at:at + 1] - mean) <= em * 1.01 + V * np.abs(mean)).all(), kind
        else:
            assert not got[:, at].any()
        y = np.abs(x - mean)
        d = e + em + V * y
        square = (terms + 3) * V * (y ** 2).mean(axis=1, keepdims=True) + (2 * y * d + d ** 2).mean(axis=1, keepdims=True)
        rel = 0.5 * square * rstd ** 2 + 4 * V
        assert (np.abs(got[:, at + 1:at + 2] / rstd - 1.0) <= rel * 1.01).all(), (kind, at, float((np.abs(got[:, at + 1:at + 2] / rstd - 1.0) / rel).max()))
