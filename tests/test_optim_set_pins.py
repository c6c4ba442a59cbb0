"""Pins for the 8-bit moments of the optimizer oracle, each against something other than itself, and the calls of
ff_adamw_set_* that are refused before a device is looked for."""
import ctypes

import numpy as np
import pytest

from oracle import optim_oracle as OO

pytest.importorskip("torch")
from paper_2608_26430_amd import binding  # noqa: E402


def test_codes_stand_for_four_significant_bits():
    for signed, top in ((True, 15 * 2.0 ** 14), (False, 15 * 2.0 ** 30)):
        u = OO.code_units(signed)
        assert u[0] == 0 and u[1] == 1 and u[15] == 15 and u[16] == 16 and u[17] == 18 and u[-1] == top
        d = np.diff(u)
        assert (d > 0).all() and (d[16:] / u[16:-1] <= 1 / 8).all() and (d[16:] / u[16:-1] >= 1 / 16).all()
        m, e = np.frexp(u[1:])
        assert (m * 16 == np.floor(m * 16)).all()


@pytest.mark.parametrize("signed", [True, False])
def test_values_on_codes_stay_and_others_go_to_a_neighbour(signed):
    rng = np.random.default_rng(1)
    u = OO.code_units(signed)
    a = rng.integers(0, u.size, 256)
    a[0] = u.size - 1                        # the block's unit is then the one below
    x = u[a] * 2.0 ** -37
    for h in (0, 65535):
        codes, exps = OO.state_codes(x, np.full(256, h), signed)
        assert np.array_equal(codes, a) and np.array_equal(OO.state_values(codes, exps, signed), x)
    y = np.abs(rng.standard_normal(700))
    y = y * np.sign(rng.standard_normal(700)) if signed else y
    codes, exps = OO.state_codes(y, rng.integers(0, 65536, 700), signed)
    got = OO.state_values(codes, exps, signed)
    assert (np.abs(got - y) <= np.maximum(np.abs(y) / 8, np.abs(y).max() * 2.0 ** -17)).all()


def test_rounding_has_no_bias_where_nearest_would_stand_still():
    """v decays by 1 - b2 a step in the mean, though that is a hundredth of the distance between two codes."""
    n, steps = 4096, 40
    v = np.full(n, 0.3)
    v[::256] = 1.0                           # keeps the unit: the others lie between codes
    cv, xv = OO.state_codes(v, np.full(n, 32768), False)
    cm, xm = np.zeros(n, np.uint8), np.zeros(n // 256, np.uint8)
    rest = np.arange(n) % 256 != 0
    start = OO.state_values(cv, xv, False)[rest].mean()
    c = np.zeros(n)
    for t in range(1, steps + 1):
        c, cm, cv, xm, xv = OO.adamw8_step(c, np.zeros(n), cm, cv, xm, xv, t, 0, 77, 0.1)
    got = OO.state_values(cv, xv, False)[rest].mean()
    # a rounding's deviation is at most half a step (v / 16); those of 40 steps and 4080 elements are independent
    assert abs(got - start * 0.999 ** steps) <= 5 * start / 16 * np.sqrt(steps / rest.sum())


def test_draws_differ_by_element_step_tensor_and_seed():
    base = OO.state_draws(1000, 3, 2, 5)
    assert (base[0] != base[1]).mean() > 0.99
    for other in (OO.state_draws(1000, 4, 2, 5), OO.state_draws(1000, 3, 1, 5), OO.state_draws(1000, 3, 2, 6)):
        assert (base[0] != other[0]).mean() > 0.99 and (base[1] != other[1]).mean() > 0.99
    assert np.array_equal(OO.state_draws(5, 3, 2, 5)[0], base[0][:5])
    assert abs(base[0].mean() / 65536 - 0.5) < 5 * np.sqrt(1 / 12 / 1000)


def test_calls_refused_on_the_host():
    lib = binding._load()
    out, p = ctypes.c_void_p(), ctypes.c_void_p(1 << 20)
    n1, arr, wd = (ctypes.c_int64 * 1)(5), (ctypes.c_void_p * 1)(1 << 20), (ctypes.c_double * 1)(0.0)
    arr_m, arr_v = (ctypes.c_void_p * 1)(2 << 20), (ctypes.c_void_p * 1)(3 << 20)

    def create(count=1, n=n1, states=0, g=0, c=arr, m=arr_m, v=arr_v, mx=None, vx=None, copy=None, wd=wd, out=ctypes.byref(out)):
        return binding._STATUS[lib.ff_adamw_set_create(count, n, states, g, c, copy, m, v, mx, vx, wd, out)]

    odd = (ctypes.c_void_p * 1)((1 << 20) + 1)
    for kw in (dict(count=0), dict(count=(1 << 20) + 1), dict(n=None), dict(states=2), dict(g=2), dict(c=None), dict(m=None),
               dict(v=None), dict(states=1), dict(c=odd), dict(m=odd), dict(copy=odd), dict(out=None),
               dict(n=(ctypes.c_int64 * 1)(-1)), dict(n=(ctypes.c_int64 * 1)(1 << 41)), dict(c=(ctypes.c_void_p * 1)(None)),
               dict(wd=(ctypes.c_double * 1)(-0.5)), dict(wd=(ctypes.c_double * 1)(float("inf")))):
        assert create(**kw) == "FF_EINVAL", kw
        assert not out
    # arrays that overlap: a tensor twice, moments that share memory, a copy inside another tensor's parameters, exponents
    two = (ctypes.c_int64 * 2)(300, 300)

    def ptrs(*a):
        return (ctypes.c_void_p * len(a))(*a)

    ok = dict(count=2, n=two, c=ptrs(0x100000, 0x101000), m=ptrs(0x102000, 0x103000), v=ptrs(0x104000, 0x105000), wd=None)
    for kw in (dict(c=ptrs(0x100000, 0x100000)), dict(c=ptrs(0x100000, 0x100000 + 1196)), dict(v=ptrs(0x102000, 0x105000)),
               dict(m=ptrs(0x102000, 0x1020a0)), dict(copy=ptrs(0x106000, 0x101004)), dict(copy=ptrs(0x106000, 0x106002))):
        assert create(**{**ok, **kw}) == "FF_EINVAL" and "overlap" in lib.ff_last_error().decode(), kw
    kw = dict(ok, states=1, mx=ptrs(0x106000, 0x106001), vx=ptrs(0x107000, 0x107002))
    assert create(**kw) == "FF_EINVAL" and "overlap" in lib.ff_last_error().decode()
    assert binding._STATUS[lib.ff_adamw_set_step(None, arr, p, None)] == "FF_EINVAL"
    assert binding._STATUS[lib.ff_adamw_set_read(None, arr, arr, None)] == "FF_EINVAL"
    lib.ff_adamw_set_destroy(None)


def test_hyperparameters_are_laid_out_as_the_header_has_them(tmp_path):
    """The binding's packed fields against the struct of include/frameft.h, compiled."""
    import os
    import shutil
    import subprocess
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    fields = ("lr", "beta1", "beta2", "eps", "grad_scale", "step", "seed", "lr_dev", "grad_scale_dev", "step_dev")
    src = tmp_path / "layout.cpp"
    src.write_text('#include <cstdio>\n#include <cstddef>\n#include "frameft.h"\nint main() {' + "".join(
        f'std::printf("%zu ", offsetof(ff_adamw_hyper, {f}));' for f in fields) + 'std::printf("%zu", sizeof(ff_adamw_hyper)); }')
    exe, root = str(tmp_path / "layout"), os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["g++", "-I" + os.path.join(root, "include"), str(src), "-o", exe], check=True, timeout=120)
    want = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True, timeout=60).stdout.split()]
    for f, at in zip(fields, want):
        one = binding._HYPER.pack(*(1 if k == f else 0 for k in fields))
        on = [i for i, b in enumerate(one) if b]
        assert on and at <= min(on) and max(on) < at + 8, f
    assert binding._HYPER.size == want[-1]
