"""Pins of the join's reference against torch and against differences, and the calls that are refused on the host."""
import ctypes

import numpy as np
import pytest

from oracle import train_oracle as TO

torch = pytest.importorskip("torch")
from paper_2608_26430_amd import binding  # noqa: E402


def _case(T, n, gate, seed=0):
    g = np.random.default_rng(seed)
    c = dict(r=g.standard_normal((T, n)), b=g.standard_normal((T, n)) * 0.7, pw=1 + 0.2 * g.standard_normal(n),
             pb=g.standard_normal(n), w=1 + 0.2 * g.standard_normal(n), bias=g.standard_normal(n))
    c["gate"] = g.standard_normal((gate, n)) if gate else None
    return c, g.standard_normal((T, n)), g.standard_normal((T, n))


def test_forward_is_torchs_layer_and_rms_norm():
    c, _, _ = _case(6, 40, 3)
    o = TO.resnorm(c["r"], c["b"], c["gate"], "layer", c["pw"], c["pb"], "rms", c["w"], None, 0.9, 1.3, 1e-6)
    t = {k: torch.from_numpy(v) for k, v in c.items()}
    p = torch.nn.functional.layer_norm(t["b"], (40,), t["pw"], t["pb"], 1e-6)
    x = 0.9 * t["r"] + 1.3 * t["gate"].repeat_interleave(2, 0) * p
    y = torch.nn.functional.rms_norm(x, (40,), t["w"], 1e-6)
    np.testing.assert_allclose(o["x"], x.numpy(), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(o["y"], y.numpy(), rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("post,norm", [("rms", "rms"), ("layer", "layer"), ("none", "layer"), ("layer", "none"), ("none", "none")])
@pytest.mark.parametrize("gate", [0, 1, 2])
def test_gradients_are_those_of_differences(post, norm, gate):
    c, dx, dy = _case(4, 9, gate)
    dy = dy if norm != "none" else None

    def value(c):
        o = TO.resnorm(c["r"], c["b"], c["gate"], post, c["pw"], c["pb"], norm, c["w"], c["bias"], 0.9, 1.3)
        return (o["x"] * dx).sum() + ((o["y"] * dy).sum() if dy is not None else 0.0)

    o = TO.resnorm(c["r"], c["b"], c["gate"], post, c["pw"], c["pb"], norm, c["w"], c["bias"], 0.9, 1.3, dx=dx, dy=dy)
    names = {"r": "dr", "b": "db", "gate": "dgate"}
    if post != "none":
        names.update(pw="dpw", pb="dpb")
    if norm != "none":
        names.update(w="dw", bias="dbias")
    for k, d in names.items():
        if c[k] is None:
            continue
        for at in [0, c[k].size // 2, c[k].size - 1]:
            lo, hi = (dict(c, **{k: c[k].copy()}) for _ in range(2))
            lo[k].flat[at] -= 1e-6
            hi[k].flat[at] += 1e-6
            assert (value(hi) - value(lo)) / 2e-6 == pytest.approx(np.ravel(o[d])[at], rel=1e-6, abs=1e-6), (k, at)


FIELDS = ("T", "n", "act", "w_dtype", "gate_dtype", "post", "norm", "post_weight", "post_bias", "weight", "bias", "gate", "ldgate",
          "groups", "res_scale", "block_scale", "post_eps", "eps")


def _packed(**d):
    return binding._RESNORM.pack(*(d.get(k, 0) for k in FIELDS))


def test_description_is_laid_out_as_the_header_has_it(tmp_path):
    """The binding's packed fields against the struct of include/frameft.h, compiled."""
    import os
    import shutil
    import subprocess
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "layout.cpp"
    src.write_text('#include <cstdio>\n#include <cstddef>\n#include "frameft.h"\nint main() {' + "".join(
        f'std::printf("%zu ", offsetof(ff_resnorm, {f}));' for f in FIELDS) + 'std::printf("%zu", sizeof(ff_resnorm)); }')
    exe = str(tmp_path / "layout")
    subprocess.run(["g++", "-I" + os.path.join(root, "include"), str(src), "-o", exe], check=True, timeout=120)
    want = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True, timeout=60).stdout.split()]
    for f, at in zip(FIELDS, want):
        one = binding._RESNORM.pack(*(1 if k == f else 0 for k in FIELDS))
        assert [i for i, b in enumerate(one) if b] and min(i for i, b in enumerate(one) if b) // 4 * 4 == at, f
    assert binding._RESNORM.size == want[-1]


def test_calls_refused_on_the_host():
    lib, p = binding._load(), ctypes.c_void_p(1 << 20)
    q = 1 << 20

    other = ctypes.c_void_p(2 << 20)

    def fwd(R=p, ldr=64, B=p, ldb=64, X=p, ldx=64, Y=other, ldy=64, stats=p, **kw):
        d = dict(T=4, n=64, act=0, w_dtype=0, gate_dtype=0, post=1, norm=1, groups=1, ldgate=64, res_scale=1.0, block_scale=1.0,
                 post_eps=1e-5, eps=1e-5)
        d.update(kw)
        return binding._STATUS[lib.ff_resnorm_fwd(_packed(**d), R, ldr, B, ldb, X, ldx, Y, ldy, stats, None)]

    bad = [dict(T=-1), dict(T=(1 << 30) + 1), dict(n=0), dict(n=(1 << 24) + 1), dict(act=2), dict(w_dtype=3), dict(gate_dtype=-1),
           dict(post=3), dict(norm=-1), dict(gate=q, groups=3), dict(gate=q, groups=0), dict(gate=q, groups=2, ldgate=63),
           dict(gate=q + 2), dict(weight=q + 1), dict(post_bias=q + 2), dict(eps=-1.0), dict(eps=float("nan")),
           dict(post_eps=float("inf")), dict(res_scale=float("nan")), dict(block_scale=float("inf")),
           dict(Y=p), dict(ldx=72), dict(R=None), dict(ldr=63), dict(B=None), dict(X=None), dict(Y=None), dict(ldy=10), dict(stats=ctypes.c_void_p(q + 4)),
           dict(R=ctypes.c_void_p(q + 2))]
    for kw in bad:
        assert fwd(**kw) == "FF_EINVAL", kw
    assert fwd(T=0, R=None) == "FF_OK"
    assert binding._STATUS[lib.ff_resnorm_fwd(None, p, 64, p, 64, p, 64, p, 64, p, None)] == "FF_EINVAL"

    def bwd(dX=p, dY=p, stats=p, dR=p, dB=other, dgate=None, dpw=None, dpb=None, dw=None, db=None, ws=p, wsn=1 << 30, lddr=64, lddb=64,
            **kw):
        d = dict(T=4, n=64, act=0, post=1, norm=1, groups=1, ldgate=64, res_scale=1.0, block_scale=1.0, post_eps=1e-5, eps=1e-5)
        d.update(kw)
        return binding._STATUS[lib.ff_resnorm_bwd(_packed(**d), p, 64, p, 64, dX, 64, dY, 64, stats, dR, lddr,
                                                  dB, lddb, 0, dgate, dpw, dpb, dw, db, ws, wsn, None)]

    for kw in (dict(dB=p), dict(lddr=72), dict(dR=None, dB=p, lddb=72), dict(dgate=p), dict(post=0, dpw=p), dict(norm=0, db=p),
               dict(dY=None), dict(stats=None),
               dict(stats=ctypes.c_void_p(q + 8)), dict(dw=p, ws=None), dict(dw=p, wsn=100), dict(dw=p, ws=ctypes.c_void_p(q + 16)),
               dict(dw=ctypes.c_void_p(q + 2)), dict(n=9001, ws=None)):
        assert bwd(**kw) == "FF_EINVAL", kw
    v = ctypes.c_int64()
    assert binding._STATUS[lib.ff_resnorm_workspace(10, 64, 3, ctypes.byref(v))] == "FF_EINVAL"
    assert binding._STATUS[lib.ff_resnorm_workspace(10, 64, 5, None)] == "FF_EINVAL"
    assert lib.ff_resnorm_workspace(10, 64, 5, ctypes.byref(v)) == 0 and v.value >= 10 * 64 * 4 * 5
