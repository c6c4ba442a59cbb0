"""Layer norm (ff_layernorm_fwd, ff_layernorm_bwd) against the fp64 reference.

Bounds per element, u the activations' unit roundoff (2^-8 for bf16, 2^-24 for fp32), v = 2^-24.  The fp32
sums over a row run over at most 32 terms per thread and 10 levels of lanes and waves, which with the
products' roundings stays under 64 v times the sum of absolute terms.  So the mean is off by at most
64 v mean|x|, h = (x - mean) rstd by e_h = 64 v (|h| + rstd (|x| + mean|x|)) (the variance's own relative error, from
the centred values' error, is of that size as well: a second 64 v |h| max_c e-ratio is covered by the factor 2
below), y by u |y| + |w| 2 e_h + 4 v (|w h| + |b|).  dx and the vectors follow by first-order propagation."""
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


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    return torch.device("cuda:0")


def _strided(a, dtype, dev, ld, at=0):
    """Tensor of a's values inside rows of ld elements, starting `at` elements into the buffer (NaN around)."""
    T, n = a.shape
    buf = torch.full((T * ld + at + 8,), float("nan"), device=dev, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    t = torch.as_strided(buf, (T, n), (ld, 1), at)
    t.copy_(torch_act(a, dtype, dev))
    return t


def _case(T, n, dtype, seed, shift=0.5):
    g = inputs.rng(seed)
    x = inputs.gaussian(g, (T, n), dtype="f32") * 1.3 + shift
    x = inputs.bf16_round(x) if dtype == "bf16" else x.astype(np.float32)
    return x, inputs.gaussian(g, (T, n), dtype=dtype), inputs.gaussian(g, (n,), std=0.3) + 1, inputs.gaussian(g, (n,))


def _bounds(x, g, w, b, u):
    y, mean, rstd = TO.layernorm_fwd(x, w, b)
    x = x.astype(np.float64)
    h = (x - mean[:, None]) * rstd[:, None]
    ax = np.abs(x).mean(axis=1, keepdims=True)
    r = rstd[:, None]
    eh = 2 * 64 * V32 * (np.abs(h) + r * (np.abs(x) + ax))
    ehm = eh.max(axis=1, keepdims=True)
    ey = u * np.abs(y) + np.abs(w) * eh + 4 * V32 * (np.abs(w * h) + np.abs(b))
    a = np.abs(g * w)
    ma, mah = a.mean(axis=1, keepdims=True), (a * np.abs(h)).mean(axis=1, keepdims=True)
    dx = TO.layernorm_bwd(x, g, w)[0]
    # the relative error of rstd is at most that of h
    rel = ehm
    edx = u * np.abs(dx) + r * ((64 * V32 + rel) * (a + ma + np.abs(h) * mah) + eh * mah + np.abs(h) * ma * ehm)
    T = x.shape[0]
    edw = (T + 64) * V32 * np.abs(g * h).sum(axis=0) + (np.abs(g) * eh).sum(axis=0)
    edb = (T + 64) * V32 * np.abs(g).sum(axis=0)
    em = 64 * V32 * ax[:, 0]
    er = rstd * (64 * V32 + ehm[:, 0])
    return y, ey, dx, edx, edw, edb, mean, em, rstd, er


def _close(got, want, bound, what):
    bad = np.abs(got - want) > bound * 1.05 + 1e-30
    assert not bad.any(), (what, int(bad.sum()), float((np.abs(got - want) / (bound + 1e-30)).max()))


# one row to many, widths of one element, of every instance (one wave with 1, 2 and 4 pieces, 4 and 16 waves), odd ones,
# and ones read three times
SIZES = [(1, 1), (3, 2), (7, 64), (1, 768), (513, 768), (130, 1000), (66, 1021), (5, 2048), (9, 2056), (600, 1024), (17, 4096),
         (33, 8192), (3, 5001), (2, 28672), (2, 32771), (3, 40000),
         (5, 9), (600, 15), (70, 2047), (40, 1025), (9, 12291), (1, 16384)]


@pytest.mark.parametrize("T,n", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layernorm_matches_oracle(dev, T, n, dtype):
    x, g, w, b = _case(T, n, dtype, 100 * T + n)
    y, ey, dx, edx, edw, edb, mean, em, rstd, er = _bounds(x, g, w, b, U[dtype])
    X, G = torch_act(x, dtype, dev), torch_act(g, dtype, dev)
    wt, bt = torch.from_numpy(w).to(dev), torch.from_numpy(b).to(dev)
    Y, m, r = ff.layernorm_fwd(X, wt, bt)
    dX, dw, db = ff.layernorm_bwd(X, G, wt, m, r)
    torch.cuda.synchronize()
    _close(to_np(Y), y, ey, "y")
    _close(to_np(m), mean, em, "mean")
    _close(to_np(r), rstd, er, "rstd")
    _close(to_np(dX), dx, edx, "dx")
    _, dwr, dbr = TO.layernorm_bwd(x, g, w)
    _close(to_np(dw), dwr, edw, "dweight")
    _close(to_np(db), dbr, edb, "dbias")
    again = ff.layernorm_bwd(X, G, wt, m, r)
    torch.cuda.synchronize()
    assert torch.equal(again[0], dX) and torch.equal(again[1], dw) and torch.equal(again[2], db)


@pytest.mark.parametrize("n,ld,at", [(1000, 1003, 1), (768, 776, 0), (768, 768, 3), (1001, 1001, 0), (9000, 9002, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_alignment_and_accumulation(dev, n, ld, at, dtype):
    """Rows inside wider ones, off 16-byte alignment, an output added to, gradients accumulated; nothing outside the rows
    is written or used (NaN there)."""
    T = 37
    x, g, w, b = _case(T, n, dtype, n + ld)
    y, ey, dx, edx, edw, edb, *_ = _bounds(x, g, w, b, U[dtype])
    gen = inputs.rng(5)
    old = inputs.gaussian(gen, (T, n), dtype=dtype)
    dw0, db0 = inputs.gaussian(gen, (n,)), inputs.gaussian(gen, (n,))
    X, G, dX, Y = (_strided(a, dtype, dev, ld, at) for a in (x, g, old, x * 0))
    wt, bt = torch.from_numpy(w).to(dev), torch.from_numpy(b).to(dev)
    _, m, r = ff.layernorm_fwd(X, wt, bt, Y=Y)
    dw, db = torch.from_numpy(dw0).to(dev), torch.from_numpy(db0).to(dev)
    ff.layernorm_bwd(X, G, wt, m, r, dX=dX, dweight=dw, dbias=db, beta_dx=0.5, accumulate=True)
    torch.cuda.synchronize()
    _close(to_np(Y), y, ey, "y")
    want = dx + 0.5 * old
    _close(to_np(dX), want, edx + U[dtype] * np.abs(want) + 4 * V32 * np.abs(old), "dx")
    _, dwr, dbr = TO.layernorm_bwd(x, g, w)
    _close(to_np(dw), dwr + dw0, edw + 2 * V32 * (np.abs(dwr) + np.abs(dw0)), "dweight")
    _close(to_np(db), dbr + db0, edb + 2 * V32 * (np.abs(dbr) + np.abs(db0)), "dbias")
    for t in (Y, dX):
        buf = torch.as_strided(t, ((T - 1) * ld + n,), (1,), t.storage_offset())
        inside = torch.zeros_like(buf, dtype=torch.bool)
        torch.as_strided(inside, (T, n), (ld, 1)).fill_(True)
        assert bool(torch.isnan(buf[~inside]).all())


def test_in_place_bf16_vectors_and_partial_outputs(dev):
    T, n = 50, 1024
    x, g, w, b = _case(T, n, "bf16", 77)
    w, b = inputs.bf16_round(w), inputs.bf16_round(b)
    y, ey, dx, edx, edw, edb, *_ = _bounds(x, g, w, b, U["bf16"])
    X, G = torch_act(x, "bf16", dev), torch_act(g, "bf16", dev)
    wt, bt = torch_act(w, "bf16", dev), torch_act(b, "bf16", dev)
    Y, m, r = ff.layernorm_fwd(X, wt, bt)
    inplace = X.clone()
    ff.layernorm_fwd(inplace, wt, bt, Y=inplace)
    only_x = ff.layernorm_bwd(X, G, wt, m, r, want_dw=False)
    only_w = ff.layernorm_bwd(X, G, wt, m, r, want_dx=False)
    both = ff.layernorm_bwd(X, G, wt, m, r)
    plain, m1, r1 = ff.layernorm_fwd(X)
    dplain = ff.layernorm_bwd(X, G, None, m1, r1, want_dw=False)[0]
    torch.cuda.synchronize()
    _close(to_np(Y), y, ey, "y")
    assert torch.equal(inplace, Y)
    assert only_x[1] is None and only_x[2] is None and only_w[0] is None
    assert torch.equal(only_x[0], both[0]) and torch.equal(only_w[1], both[1]) and torch.equal(only_w[2], both[2])
    _close(to_np(both[0]), dx, edx, "dx")
    one, zero = np.ones(n), np.zeros(n)
    yp, eyp, dxp, edxp, *_ = _bounds(x, g, one, zero, U["bf16"])
    _close(to_np(plain), yp, eyp, "y without weight")
    _close(to_np(dplain), dxp, edxp, "dx without weight")


def test_large_mean_and_constant_rows(dev):
    """A mean a thousand times the spread keeps its digits (the variance is the centred row's); a constant row gives the
    bias, and its gradient is finite; a NaN stays in its row."""
    n = 768
    x, g, w, b = _case(6, n, "f32", 3, shift=0.0)
    x = (x + np.float32(1000.0)).astype(np.float32)
    x[2] = 3.0
    x[4, 5] = np.nan
    X, G = torch_act(x, "f32", dev), torch_act(g, "f32", dev)
    wt, bt = torch.from_numpy(w).to(dev), torch.from_numpy(b).to(dev)
    Y, m, r = ff.layernorm_fwd(X, wt, bt)
    dX = ff.layernorm_bwd(X, G, wt, m, r, want_dw=False)[0]
    torch.cuda.synchronize()
    rows = [0, 1, 3, 5]
    y, ey, dx, edx, *_ = _bounds(x[rows], g[rows], w, b, U["f32"])
    _close(to_np(Y)[rows], y, ey, "y")
    _close(to_np(dX)[rows], dx, edx, "dx")
    assert np.array_equal(to_np(Y)[2], b.astype(np.float64))
    assert np.isfinite(to_np(dX)[2]).all()
    assert np.isnan(to_np(Y)[4]).all() and np.isfinite(to_np(Y)[rows]).all()


def test_no_rows(dev):
    X = torch.empty((0, 64), device=dev)
    Y, m, r = ff.layernorm_fwd(X)
    dw, db = torch.ones(64, device=dev), torch.ones(64, device=dev)
    dX, _, _ = ff.layernorm_bwd(X, X, None, m, r, dweight=dw, dbias=db, accumulate=True)
    assert Y.shape == (0, 64) and dX.shape == (0, 64) and bool((dw == 1).all())
    ff.layernorm_bwd(X, X, None, m, r, dweight=dw, dbias=db)
    torch.cuda.synchronize()
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_refusals(dev):
    X = torch.zeros((4, 64), device=dev)
    Y, m, r = ff.layernorm_fwd(X)
    w = torch.ones(64, device=dev)
    for bad in (lambda: ff.layernorm_fwd(X.t()), lambda: ff.layernorm_fwd(X, w[:32]), lambda: ff.layernorm_fwd(X.cpu()),
                lambda: ff.layernorm_fwd(X, w, w.bfloat16()), lambda: ff.layernorm_fwd(X, Y=X.bfloat16()),
                lambda: ff.layernorm_bwd(X, X[:2], w, m, r), lambda: ff.layernorm_bwd(X, X, w, m[:2], r),
                lambda: ff.layernorm_bwd(X, X, w, m, r, beta_dx=1.0), lambda: ff.layernorm_bwd(X, X, w, m, r, accumulate=True)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        ff.layernorm_fwd(X.half())
    with pytest.raises(ff.FrameFTError):
        ff.layernorm_bwd(X, X, w, m, r, workspace=torch.empty(64, dtype=torch.uint8, device=dev))


@pytest.mark.parametrize("n", [9, 1021, 2047, 5473])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_odd_widths_in_place(dev, n, dtype):
    """The last piece of an odd row overlaps the one before it: in place, the same bits as into another tensor."""
    x, g, w, b = _case(300, n, dtype, n)
    X, wt, bt = torch_act(x, dtype, dev), torch.from_numpy(w).to(dev), torch.from_numpy(b).to(dev)
    Y = ff.layernorm_fwd(X, wt, bt)[0]
    got = X.clone()
    ff.layernorm_fwd(got, wt, bt, Y=got)
    torch.cuda.synchronize()
    assert torch.equal(got, Y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_rows_than_one_launch_has_workgroups_for(dev, dtype):
    """Rows narrower than a 16-byte piece, 2^22 and a few of them: a workgroup each would be more threads than a launch can
    have."""
    T, n = (1 << 22) + 5, 3
    x, g, w, b = _case(T, n, dtype, 11)
    X, G = torch_act(x, dtype, dev), torch_act(g, dtype, dev)
    wt, bt = torch.from_numpy(w).to(dev), torch.from_numpy(b).to(dev)
    Y, m, r = ff.layernorm_fwd(X, wt, bt)
    dX, dw, db = ff.layernorm_bwd(X, G, wt, m, r)
    torch.cuda.synchronize()
    rows = np.r_[0:500, (1 << 20) - 250:(1 << 20) + 250, (1 << 21) - 5:(1 << 21) + 5, T - 500:T]
    y, ey, dx, edx, _, _, mean, em, rstd, er = _bounds(x[rows], g[rows], w, b, U[dtype])
    at = torch.from_numpy(rows).to(dev)
    for got, want, bound, what in ((Y, y, ey, "y"), (m, mean, em, "mean"), (r, rstd, er, "rstd"), (dX, dx, edx, "dx")):
        _close(to_np(got[at]), want, bound, what)
    assert bool(torch.isfinite(Y).all()) and bool(torch.isfinite(dX).all())
    # at most T / 256 terms a workgroup's thread adds, then the partial rows: below (T / 256 + 1024) v of the absolute sums
    y64, mean64, rstd64 = TO.layernorm_fwd(x, w, b)
    h = (x.astype(np.float64) - mean64[:, None]) * rstd64[:, None]
    eh = 2 * 64 * V32 * (np.abs(h) + rstd64[:, None] * (np.abs(x) + np.abs(x).mean(axis=1, keepdims=True)))
    terms = (T / 256 + 1024) * V32
    _close(to_np(dw), (g * h).sum(axis=0), terms * np.abs(g * h).sum(axis=0) + (np.abs(g) * eh).sum(axis=0), "dweight")
    _close(to_np(db), g.astype(np.float64).sum(axis=0), terms * np.abs(g).astype(np.float64).sum(axis=0), "dbias")


# more rows than the kernels have places for at once, three times over and a few: rows of one wave (4096 places forward, 2048
# backward) and of eight (1024; 512, above 4096 wide 256), whole pieces and a last one that overlaps
@pytest.mark.parametrize("T,n", [(12609, 768), (12609, 1021), (12300, 2047), (3100, 2056), (3100, 8192), (3100, 5473)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_workgroups_walk_over_rows(dev, T, n, dtype):
    """Every row of a long call has the bits that it has in a short one, whose workgroups take one row each; in place, added to
    an old gradient; dw and db, kept over the rows of a workgroup, against the reference: at most T / 256 rows a thread, 4 waves,
    then 16 partial rows a thread and 32 of those, below (T / 256 + 128) v of the absolute sums and what h is off."""
    x, g, w, b = _case(T, n, dtype, T + n)
    X, G = torch_act(x, dtype, dev), torch_act(g, dtype, dev)
    wt, bt = torch.from_numpy(w).to(dev), torch.from_numpy(b).to(dev)
    old = torch_act(inputs.gaussian(inputs.rng(n), (T, n), dtype=dtype), dtype, dev)
    Y, m, r = ff.layernorm_fwd(X, wt, bt)
    inplace = X.clone()
    _, m2, r2 = ff.layernorm_fwd(inplace, wt, bt, Y=inplace)
    dX, dw, db = ff.layernorm_bwd(X, G, wt, m, r)
    onto = old.clone()
    dw2, db2 = dw.clone(), db.clone()
    ff.layernorm_bwd(X, G, wt, m, r, dX=onto, dweight=dw2, dbias=db2, beta_dx=0.5, accumulate=True)
    torch.cuda.synchronize()
    assert torch.equal(inplace, Y) and torch.equal(m2, m) and torch.equal(r2, r)
    assert torch.equal(dw2, 2 * dw) and torch.equal(db2, 2 * db)
    for t in range(0, T, 250):
        s = slice(t, min(T, t + 250))
        y, ms, rs = ff.layernorm_fwd(X[s], wt, bt)
        dx = ff.layernorm_bwd(X[s], G[s], wt, ms, rs, want_dw=False)[0]
        dx2 = ff.layernorm_bwd(X[s], G[s], wt, ms, rs, dX=old[s].clone(), beta_dx=0.5, want_dw=False)[0]
        for short, long in ((y, Y), (ms, m), (rs, r), (dx, dX), (dx2, onto)):
            assert torch.equal(short, long[s]), t
    y, mean, rstd = TO.layernorm_fwd(x, w, b)
    h = (x.astype(np.float64) - mean[:, None]) * rstd[:, None]
    eh = 2 * 64 * V32 * (np.abs(h) + rstd[:, None] * (np.abs(x) + np.abs(x).mean(axis=1, keepdims=True)))
    terms = (T / 256 + 128) * V32
    _close(to_np(dw), (g * h).sum(axis=0), terms * np.abs(g * h).sum(axis=0) + (np.abs(g) * eh).sum(axis=0), "dweight")
    _close(to_np(db), g.astype(np.float64).sum(axis=0), terms * np.abs(g).astype(np.float64).sum(axis=0), "dbias")
    rows = np.r_[0:40, T // 2:T // 2 + 40, T - 40:T]
    y, ey, dx, edx, _, _, mean, em, rstd, er = _bounds(x[rows], g[rows], w, b, U[dtype])
    at = torch.from_numpy(rows).to(dev)
    for got, want, bound, what in ((Y, y, ey, "y"), (m, mean, em, "mean"), (r, rstd, er, "rstd"), (dX, dx, edx, "dx")):
        _close(to_np(got[at]), want, bound, what)
