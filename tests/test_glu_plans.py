"""Which kernels, tiles and splits the sizes of test_gpu_glu.py run (csrc/glu_plan.h, compiled and asked on the CPU), so that a change
of a cost table cannot take a kernel out of the tests unnoticed; and the calls that are refused on the host."""
import ctypes
import os
import shutil
import subprocess

import pytest

pytest.importorskip("torch")
from paper_2608_26430_amd import binding  # noqa: E402
from tests.test_gpu_glu import BIG, SIZES  # noqa: E402

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LARGE, MEDIUM, SMALL = 0, 1, 2


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("plans") / "glu_plans")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2608_26430_amd", "csrc"), os.path.join(HERE, "plans", "glu_plans.cpp"),
                    "-o", exe], check=True, timeout=300)

    def ask(T, n, F, bf16):
        out = subprocess.run([exe], input=f"{T} {n} {F} {int(bf16)}\n", capture_output=True, text=True, check=True, timeout=60).stdout
        w = [int(x) for x in out.split()]       # ("gap": not a number)
        plan = {}
        for name, rows in (("proj", T), ("dx", T), ("dw", F)):
            parts = [dict(zip(("rows", "tile", "ks", "splits", "tiles", "rest"), [w.pop(0) for _ in range(6)]))
                     for _ in range(w.pop(0))]
            assert sum(p["rows"] for p in parts) == rows
            plan[name] = parts
        return plan

    return ask


@pytest.mark.parametrize("bf16", [True, False])
def test_sizes_run_every_kernel(plans, bf16):
    p = [plans(*s, bf16) for s in SIZES + (BIG if bf16 else [])]
    proj = [q for x in p for q in x["proj"]]
    # few tokens and few columns: 16 and 32 tokens a workgroup, with each number of waves that both run, and several groups of tokens
    few = {(q["ks"], q["rows"] > 16) for q in proj if q["ks"]}
    assert few == {(4, False), (8, False), (4, True), (8, True)}, few
    assert any(q["ks"] and q["rows"] > 32 for q in proj)
    tiles = {MEDIUM, SMALL} | ({LARGE} if bf16 else set())
    assert {q["tile"] for q in proj if not q["ks"]} == tiles
    for k in ("dx", "dw"):
        parts = [q for x in p for q in x[k]]
        assert {q["tile"] for q in parts} == tiles, k
        assert {q["splits"] > 1 for q in parts} == {True, False}
    for k in ("proj", "dx", "dw") if bf16 else ():
        # large tiles, more of them than workgroups, and halved ones; calls in two parts
        assert any(q["tile"] == LARGE and q["tiles"] > 256 and not q["ks"] for x in p for q in x[k]), k
        assert any(q["rest"] and not q["ks"] for x in p for q in x[k]), k
        assert any(q["rest"] == q["tiles"] and not q["ks"] for x in p for q in x[k]), k
        assert any(len(x[k]) == 2 for x in p), k


@pytest.mark.parametrize("T,n,F", [(1 << 28, 8, 8), (1 << 28, 8, 64), (1 << 28, 64, 8), (1 << 26, 8, 512), (1 << 20, 8, 1 << 16),
                                   (4, 1 << 18, 1 << 18), (1 << 18, 1 << 18, 64)])
@pytest.mark.parametrize("bf16", [True, False])
def test_largest_calls_fit_their_launches(plans, T, n, F, bf16):
    """Workgroups times threads stay below 2^32, and tile numbers in 31 bits, at the longest calls that a card's memory holds."""
    p = plans(T, n, F, bf16)
    for name in p:
        for q in p[name]:
            if q["ks"]:
                groups = -(-F // 16) * -(-q["rows"] // 32)
                assert groups * q["ks"] * 64 < 2 ** 32
            else:
                assert q["tiles"] < 2 ** 31 and (q["tile"] == LARGE or q["tiles"] * 256 < 2 ** 32), (name, q)


def test_deep_tiles_of_dx_are_run(plans):
    """Medium tiles with four buffers, of split sums and of whole ones, with a last k tile that is not full."""
    deep = set()
    for T, n, F in SIZES:
        for q in plans(T, n, F, True)["dx"]:
            per = -(-(-(-F // 64)) // q["splits"])
            if q["tile"] == MEDIUM and q["tiles"] <= 256 and 2 * per >= 12 and F % 64:
                deep.add(q["splits"] > 1)
    assert deep == {True, False}


def test_calls_refused_on_the_host():
    lib, q = binding._load(), 1 << 20
    p = ctypes.c_void_p(q)

    def fwd(T=4, n=64, F=32, act=1, fn=0, X=p, ldx=64, Wg=p, Wu=p, ldw=64, Ag=None, Au=None, lda=32, H=p, ldh=32, G=None, U=None, ldg=32):
        return binding._STATUS[lib.ff_glu_fwd(T, n, F, act, fn, X, ldx, Wg, Wu, ldw, Ag, Au, lda, H, ldh, G, U, ldg, None)]

    def at(i):
        return ctypes.c_void_p(q + (i << 12))

    odd = ctypes.c_void_p(q + 8)
    for kw in (dict(T=-1), dict(T=(1 << 28) + 1), dict(n=60), dict(n=0), dict(F=36), dict(F=(1 << 18) + 8), dict(act=2), dict(fn=3),
               dict(fn=-1), dict(X=None), dict(ldx=56), dict(ldx=68), dict(ldx=(1 << 20) + 8), dict(Wg=None), dict(Wu=odd), dict(ldw=60),
               dict(Ag=odd), dict(Au=p, lda=24), dict(H=None), dict(ldh=36), dict(G=p), dict(U=p), dict(G=p, U=p, ldg=24),
               dict(G=p, U=at(9)), dict(G=at(9), U=at(9))):
        assert fwd(**kw) == "FF_EINVAL", kw
    assert fwd(T=0, X=None, H=None) == "FF_OK"

    def bwd(T=4, dH=at(1), X=p, Wg=p, Wu=p, G=at(2), U=at(3), dG=at(4), dU=at(5), dX=at(6), dWg=None, dWu=None, lddw=64, lddg=32,
            ws=p, wsn=1 << 30):
        return binding._STATUS[lib.ff_glu_bwd(T, 64, 32, 1, 0, dH, 32, X, 64, Wg, Wu, 64, None, None, 32, G, U, 32, dG, dU, lddg, 0.0,
                                              dX, 64, 0.0, dWg, dWu, lddw, ws, wsn, None)]

    for kw in (dict(dU=at(4)), dict(dG=at(1), lddg=40), dict(dU=at(2), lddg=40), dict(dG=at(2), lddg=40), dict(dWg=at(7), dWu=at(7)),
               dict(dH=None), dict(G=None), dict(U=None), dict(G=None, U=None, X=None), dict(dG=None), dict(dU=odd), dict(dX=odd),
               dict(dWg=p), dict(dWg=p, dWu=p, X=None), dict(Wg=None), dict(dWg=p, dWu=p, lddw=60), dict(ws=None),
               dict(ws=ctypes.c_void_p(q + 16)), dict(wsn=0)):
        assert bwd(**kw) == "FF_EINVAL", kw
    assert bwd(T=0, dH=None, dG=None, dX=None) == "FF_OK"
    v = ctypes.c_int64()
    for a in ((4, 64, 32, 1, 4), (4, 64, 32, 1, -1), (4, 63, 32, 1, 1), (4, 64, 32, 3, 1)):
        assert binding._STATUS[lib.ff_glu_workspace(*a, ctypes.byref(v))] == "FF_EINVAL"
    assert binding._STATUS[lib.ff_glu_workspace(4, 64, 32, 1, 3, None)] == "FF_EINVAL"
