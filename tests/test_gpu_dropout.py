"""Dropout (ff_dropout) against the fp64 reference: the mask exactly, kept values within the roundings (scaling in fp32
by a factor rounded once: 2 v, the residual's addition: v, the result to the activations' type: u)."""
import numpy as np
import pytest

from oracle import train_oracle as TO
from paper_2608_26430_amd import inputs
from tests.parity_util import to_np, torch_act

torch = pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402

pytestmark = pytest.mark.gpu
V32 = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
SEED = 0xFEDCBA9876543210


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    return torch.device("cuda:0")


def _check(Y, x, p, seed, offset, dtype, res=None):
    want = TO.dropout(x, p, seed, offset, res)
    scaled = TO.dropout(np.abs(x), p, seed, offset)
    bound = U[dtype] * np.abs(want) + 4 * V32 * (scaled + (0 if res is None else np.abs(res)))
    got = to_np(Y)
    assert np.all(np.abs(got - want) <= bound)
    if res is None:     # no activation is zero, so zeros are the dropped elements
        np.testing.assert_array_equal(got != 0, TO.dropout_mask(*x.shape, p, seed, offset))


@pytest.mark.parametrize("T,n,ld,at", [(1, 1, 1, 0), (5, 7, 7, 0), (64, 256, 256, 0), (33, 1001, 1001, 0), (33, 1001, 1008, 0),
                                       (40, 512, 515, 1), (300, 4096, 4096, 0), (9, 28672, 28680, 8), (3000, 9, 9, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout_matches_oracle(dev, T, n, ld, at, dtype, residual):
    g = inputs.rng(T * n + ld)
    x, r = inputs.gaussian(g, (T, n), dtype=dtype), inputs.gaussian(g, (T, n), dtype=dtype)
    x[x == 0] = 1.0
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def place(a):
        buf = torch.full((T * ld + at + 8,), float("nan"), device=dev, dtype=tdt)
        t = torch.as_strided(buf, (T, n), (ld, 1), at)
        t.copy_(torch_act(a, dtype, dev))
        return t, buf

    (X, _), (R, _), (Y, ybuf) = place(x), place(r), place(x * 0)
    got = ff.dropout(X, 0.25, SEED, 77, residual=R if residual else None, Y=Y)
    torch.cuda.synchronize()
    assert got is Y
    _check(Y, x, 0.25, SEED, 77, dtype, r.astype(np.float64) if residual else None)
    inside = torch.zeros_like(ybuf, dtype=torch.bool)
    torch.as_strided(inside, (T, n), (ld, 1), at).fill_(True)
    assert bool(torch.isnan(ybuf[~inside]).all())


@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.5, 0.999999, 1.0])
def test_shares(dev, p):
    x = inputs.gaussian(inputs.rng(4), (100, 640))
    x[x == 0] = 1.0
    X = torch_act(x, "f32", dev)
    Y = ff.dropout(X, p, 3, 9)
    torch.cuda.synchronize()
    _check(Y, x, p, 3, 9, "f32")
    if p == 0.0:
        assert torch.equal(Y, X)


def test_forward_and_backward_masks_agree_in_place_and_across_types(dev):
    T, n = 70, 1000
    g = inputs.rng(6)
    x, up = inputs.gaussian(g, (T, n), dtype="bf16"), inputs.gaussian(g, (T, n), dtype="bf16")
    x[x == 0] = 1.0
    up[up == 0] = 1.0
    X, G = torch_act(x, "bf16", dev), torch_act(up, "f32", dev)
    Y = ff.dropout(X, 0.4, 11, 5)
    dX = ff.dropout(G, 0.4, 11, 5)
    inplace = X.clone()
    ff.dropout(inplace, 0.4, 11, 5, Y=inplace)
    onto = X.clone()
    ff.dropout(X, 0.4, 11, 5, residual=onto, Y=onto)
    want = ff.dropout(X, 0.4, 11, 5, residual=X)
    torch.cuda.synchronize()
    assert torch.equal(Y != 0, dX != 0) and torch.equal(inplace, Y) and torch.equal(onto, want)


def test_dropped_nan_and_infinity_are_zero(dev):
    X = torch.full((32, 96), float("nan"), device=dev)
    X[::2] = float("inf")
    Y = ff.dropout(X, 0.5, 1, 2)
    torch.cuda.synchronize()
    keep = torch.from_numpy(TO.dropout_mask(32, 96, 0.5, 1, 2)).to(dev)
    assert bool((Y[~keep] == 0).all()) and not bool(torch.isfinite(Y[keep]).any())


def test_device_offset_and_graph_replays(dev):
    """A captured call draws the mask of offset + the device's value at every replay."""
    x = inputs.gaussian(inputs.rng(8), (40, 328))
    x[x == 0] = 1.0
    X = torch_act(x, "f32", dev)
    Y = torch.empty_like(X)
    step = torch.zeros(1, dtype=torch.int64, device=dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ff.dropout(X, 0.3, SEED, 100, Y=Y, offset_dev=step)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ff.dropout(X, 0.3, SEED, 100, Y=Y, offset_dev=step)
    for k in (0, 1, 2, 1 << 33):
        step.fill_(k)
        Y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _check(Y, x, 0.3, SEED, 100 + k, "f32")


def test_stream_argument(dev):
    x = inputs.gaussian(inputs.rng(9), (64, 512))
    X = torch_act(x, "f32", dev)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    Y = ff.dropout(X, 0.3, 5, 6, stream=s)
    s.synchronize()
    assert torch.equal(Y, ff.dropout(X, 0.3, 5, 6))


def test_refusals(dev):
    X = torch.zeros((4, 64), device=dev)
    for bad in (lambda: ff.dropout(X.t(), 0.1, 1), lambda: ff.dropout(X.cpu(), 0.1, 1), lambda: ff.dropout(X, 0.1, 1, Y=X[:2]),
                lambda: ff.dropout(X, 0.1, 1, residual=X.bfloat16()),
                lambda: ff.dropout(X, 0.1, 1, offset_dev=torch.zeros(1, device=dev))):
        with pytest.raises(ValueError):
            bad()
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(ff.FrameFTError):
            ff.dropout(X, p, 1)
    assert ff.dropout(X[:0], 0.1, 1).shape == (0, 64)


@pytest.mark.parametrize("T,n,dtype,residual", [(2100, 28675, "bf16", True), (2100, 28675, "f32", False), (1 << 20, 17, "f32", True),
                                                (1 << 20, 17, "bf16", False), (70_000, 500, "bf16", True)])
def test_more_blocks_than_threads(dev, T, n, dtype, residual):
    """More than 2^21 blocks of eight: a thread takes several, carrying row and column along.  Rows from the start, around
    every seam between two turns, some in between and the end, against the reference."""
    nb = -(-n // 8)
    assert T * nb > 1 << 21
    g = inputs.rng(T + n)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device=dev)
    gen.manual_seed(n)
    X = (torch.rand((T, n), generator=gen, device=dev) + 0.5).to(tdt)
    R = torch.randn((T, n), generator=gen, device=dev).to(tdt) if residual else None
    Y = ff.dropout(X, 0.3, SEED, 5, residual=R)
    torch.cuda.synchronize()
    seams = [k * (1 << 21) // nb for k in range(1, T * nb // (1 << 21) + 1)]
    rows = np.unique(np.clip(np.r_[0:3, [s + d for s in seams for d in (-1, 0, 1)], g.integers(0, T, 30), T - 3:T], 0, T - 1))
    block = rows[:, None].astype(np.uint64) * np.uint64(nb) + np.arange(nb, dtype=np.uint64)
    counter = np.zeros(block.shape + (4,), dtype=np.uint64)
    counter[..., 0], counter[..., 1], counter[..., 2] = block & np.uint64(0xFFFFFFFF), block >> np.uint64(32), 5
    words = TO.philox4x32(counter, (SEED & 0xFFFFFFFF, SEED >> 32)).astype(np.int64)
    draws = np.stack([words & 0xFFFF, words >> 16], axis=-1).reshape(len(rows), nb * 8)[:, :n]
    drop = TO.dropout_draws(0.3)
    at = torch.from_numpy(rows).to(dev)
    scaled = np.where(draws >= drop, to_np(X[at]) * (65536 / (65536 - drop)), 0.0)
    want = scaled + (to_np(R[at]) if residual else 0.0)
    bound = U[dtype] * np.abs(want) + 4 * V32 * (scaled + (np.abs(to_np(R[at])) if residual else 0.0))
    got = to_np(Y[at])
    assert np.all(np.abs(got - want) <= bound)
    if not residual:
        np.testing.assert_array_equal(got != 0, draws >= drop)
        # the whole result: the share that is kept, within six standard deviations
        kept = float((Y != 0).double().mean())
        assert abs(kept - (1 - drop / 65536)) <= 6 * (0.21 / (T * n)) ** 0.5
