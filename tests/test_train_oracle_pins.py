"""The fp64 references of layer norm, dropout and the head's loss: gradients against central differences,
Philox against its published known answers, and the entry points' checks that need no device."""
import ctypes

import numpy as np
import pytest

from oracle import train_oracle as TO
from paper_2608_26430_amd import binding, inputs


def _diff(f, x, h=1e-5):
    """Central differences of the scalar f at x."""
    out = np.empty_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = f(x)
        x[i] = keep - h
        out[i] = (up - f(x)) / (2 * h)
        x[i] = keep
    return out


def test_philox_known_answers():
    """The three vectors published with the generator (counter and key of zeros, of ones, of pi's digits)."""
    cases = [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
             ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
             ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
              (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]
    for counter, key, want in cases:
        got = TO.philox4x32(np.array([counter], dtype=np.uint64), key)[0]
        assert tuple(int(w) for w in got) == want


def test_layernorm_gradient_is_the_differences():
    g = inputs.rng(1)
    x, up, w, b = g.standard_normal((3, 7)), g.standard_normal((3, 7)), g.standard_normal(7), g.standard_normal(7)
    f = lambda x, w, b: float((TO.layernorm_fwd(x, w, b)[0] * up).sum())
    dx, dw, db = TO.layernorm_bwd(x, up, w)
    np.testing.assert_allclose(dx, _diff(lambda v: f(v, w, b), x.copy()), atol=1e-8)
    np.testing.assert_allclose(dw, _diff(lambda v: f(x, v, b), w.copy()), atol=1e-8)
    np.testing.assert_allclose(db, _diff(lambda v: f(x, w, v), b.copy()), atol=1e-8)


def test_xent_gradient_is_the_differences():
    g = inputs.rng(2)
    H, W = g.standard_normal((5, 4)), g.standard_normal((6, 4))
    target, dloss = np.array([0, 5, -100, 3, 6]), g.standard_normal(5)
    loss, lse, dH, dW, _ = TO.xent(H, W, target, dloss, 0.7, rows=2)
    assert loss[2] == 0 and loss[4] == 0 and np.all(dH[[2, 4]] == 0)
    z = H @ W.T
    np.testing.assert_allclose(lse, np.log(np.exp(z).sum(axis=1)), rtol=1e-12)
    f = lambda H, W: float((TO.xent(H, W, target)[0] * dloss * 0.7).sum())
    np.testing.assert_allclose(dH, _diff(lambda v: f(v, W), H.copy()), atol=1e-8)
    np.testing.assert_allclose(dW, _diff(lambda v: f(H, v), W.copy()), atol=1e-8)


def test_dropout_mask_keeps_its_share_and_depends_on_every_argument():
    base = TO.dropout_mask(64, 1001, 0.3, 12345, 7)
    share = 1 - base.mean()
    # binomial standard deviation of 64,064 draws: 0.0018
    assert abs(share - 0.3) < 5 * 0.0018
    assert not TO.dropout_mask(3, 5, 1.0, 1).any() and TO.dropout_mask(3, 5, 0.0, 1).all()
    for seed, offset in ((12346, 7), (12345, 8), (12345 + (1 << 32), 7), (12345, 7 + (1 << 32))):
        other = TO.dropout_mask(64, 1001, 0.3, seed, offset)
        # independent masks agree on 0.58 of the elements
        assert abs((other == base).mean() - 0.58) < 5 * 0.002


# ------------------------------------------------------------------ checks that precede device use

def _status(code):
    return binding._STATUS[code]


def test_layernorm_refusals_without_a_device():
    lib, p = binding._load(), ctypes.c_void_p(4096)
    fwd = lambda T=4, n=8, act=0, X=p, ldx=8, wt=0, w=None, eps=1e-5, Y=p, ldy=8: _status(
        lib.ff_layernorm_fwd(T, n, act, X, ldx, wt, w, None, eps, Y, ldy, None, None, None))
    for bad in (dict(T=-1), dict(n=0), dict(act=2), dict(wt=2), dict(X=None), dict(Y=None), dict(ldx=7), dict(ldy=7),
                dict(eps=-1.0), dict(eps=float("nan")), dict(X=ctypes.c_void_p(4098)), dict(w=ctypes.c_void_p(4097))):
        assert fwd(**bad) == "FF_EINVAL", bad
    assert fwd(T=0, X=None, Y=None) == "FF_OK"
    bwd = lambda T=4, n=8, G=p, mean=p, dX=p, dw=p, ws=p, wsn=1 << 20, lddx=8: _status(
        lib.ff_layernorm_bwd(T, n, 0, p, 8, G, 8, 0, None, mean, p, 0.0, dX, lddx, 0, dw, None, ws, wsn, None))
    for bad in (dict(G=None), dict(mean=None), dict(ws=None), dict(wsn=8), dict(lddx=4), dict(ws=ctypes.c_void_p(4100)),
                dict(dw=ctypes.c_void_p(4097)), dict(T=-2)):
        assert bwd(**bad) == "FF_EINVAL", bad
    assert bwd(dX=None, dw=None, ws=None, wsn=0) == "FF_OK"      # nothing wanted


def test_dropout_refusals_without_a_device():
    lib, p = binding._load(), ctypes.c_void_p(4096)
    call = lambda T=4, n=8, act=0, X=p, ldx=8, q=0.1, od=None, R=None, ldr=8, Y=p, ldy=8: _status(
        lib.ff_dropout(T, n, act, X, ldx, q, 1, 2, od, R, ldr, Y, ldy, None))
    for bad in (dict(T=-1), dict(n=0), dict(act=7), dict(X=None), dict(Y=None), dict(q=-0.1), dict(q=1.5),
                dict(q=float("nan")), dict(ldx=3), dict(R=p, ldr=2), dict(od=ctypes.c_void_p(4100)),
                dict(Y=ctypes.c_void_p(4097))):
        assert call(**bad) == "FF_EINVAL", bad
    assert call(T=0, X=None) == "FF_OK"


def test_xent_refusals_without_a_device():
    lib, p = binding._load(), ctypes.c_void_p(4096)
    need = ctypes.c_int64()
    assert _status(lib.ff_xent_workspace(4, 16, 100, 1, 3, ctypes.byref(need))) == "FF_OK"
    step = lambda T=4, n=16, V=100, act=1, H=p, ldh=16, W=p, ldw=16, tgt=p, loss=p, lse=p, dH=p, lddh=16, dW=p, lddw=16, \
        ws=p, wsn=need.value: _status(lib.ff_xent_step(T, n, V, act, H, ldh, W, ldw, tgt, None, 1.0, loss, lse, 0.0, dH, lddh,
                                                       0.0, dW, lddw, ws, wsn, None))
    odd = ctypes.c_void_p(4104)
    for bad in (dict(T=-1), dict(n=12), dict(n=0), dict(V=0), dict(act=3), dict(H=None), dict(W=None), dict(tgt=None),
                dict(loss=None), dict(lse=None), dict(ldh=8), dict(ldh=20), dict(ldw=(1 << 20) + 8), dict(H=odd), dict(W=odd),
                dict(dH=odd), dict(dW=odd), dict(lddh=12), dict(lddw=8), dict(ws=None), dict(ws=odd), dict(wsn=need.value - 1),
                dict(tgt=ctypes.c_void_p(4100))):
        assert step(**bad) == "FF_EINVAL", bad
    assert _status(lib.ff_xent_workspace(4, 16, 100, 1, 4, ctypes.byref(need))) == "FF_EINVAL"
    assert _status(lib.ff_xent_workspace(4, 16, 100, 1, 3, None)) == "FF_EINVAL"
    assert _status(lib.ff_xent_fwd(4, 16, 100, 1, p, 16, p, 16, p, None, p, p, 1 << 30, None)) == "FF_EINVAL"
    assert _status(lib.ff_xent_bwd(4, 16, 100, 1, p, 16, p, 16, p, None, None, None, 1.0, 0.0, p, 16, 0.0, None, 0, p, 1 << 30,
                                   None)) == "FF_EINVAL"


@pytest.mark.parametrize("T,V,act", [(4096, 32000, 1), (100_000, 128_000, 1), (3000, 1_000_000, 0), (1, 2, 1)])
def test_xent_workspace_is_bounded(T, V, act):
    """P of one piece (256 MiB, or 256 tokens), statistics, and sums of a piece's dH, however many tokens there are."""
    n = 512
    lib, v = binding._load(), ctypes.c_int64()
    assert lib.ff_xent_workspace(T, n, V, act, 1, ctypes.byref(v)) == 0
    esz = 2 if act else 4
    piece = max(256 << 20, 256 * (V + 64) * esz)
    rows = min(T, max(256, piece // (V * esz)))
    assert v.value <= piece + max(64 << 20, 256 * (V // 4 + 16)) + 64 * rows * n * 4 + rows * (V // 4 + 16) + 8192
