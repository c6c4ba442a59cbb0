"""Which tiles, walks and pieces the sizes of test_gpu_xent_tiles.py run: the plan of a call (csrc/xent_plan.h), compiled and asked
on the CPU, so that a change of its cost table cannot take a kernel out of the tests unnoticed."""
import os
import shutil
import subprocess

import pytest

pytest.importorskip("torch")
from tests.test_gpu_xent_tiles import CASES, LARGE  # noqa: E402

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("plans") / "loss_plans")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2608_26430_amd", "csrc"), os.path.join(HERE, "plans", "loss_plans.cpp"),
                    "-o", exe], check=True, timeout=300)

    def ask(T, n, V, dtype, dh, dw):
        line = f"{T} {n} {V} {int(dtype == 'bf16')} {int(dh)} {int(dw)}\n"
        w = subprocess.run([exe], input=line, capture_output=True, text=True, check=True, timeout=60).stdout.split()
        out = {}
        while w:
            name = w.pop(0)
            count = 3 if name in ("logits", "dh", "dw") else 1      # tile, split, tiles
            out[name] = tuple(int(w.pop(0)) for _ in range(count)) if count > 1 else int(w.pop(0))
        return out

    return ask


@pytest.mark.parametrize("T,n,V,dtype,dh,dw,want", CASES)
def test_large_cases_run_what_they_are_there_for(plan, T, n, V, dtype, dh, dw, want):
    p = plan(T, n, V, dtype, dh, dw)
    for product in ("logits", "dh", "dw"):
        if product in want:
            assert p[product][0] == want[product], (product, p)
    for product in want.get("walks", "").split():
        assert p[product][0] == LARGE and p[product][2] > 256, (product, p)
    if "split" in want:
        assert p["dh"][1] == want["split"], p
    if "pieces" in want:
        pieces = -(-V // p["Vp"]) if p["by_vocab"] else -(-T // p["Tp"])
        assert pieces == want["pieces"], p
    alone = plan(T, n, V, dtype, False, False)
    assert -(-T // alone["Tf"]) == want["forwards"] and alone["Tf"] == p["Tf"]


def test_every_product_has_a_case_on_large_tiles_that_walks():
    for product in ("logits", "dh", "dw"):
        assert any(product in c[6].get("walks", "").split() for c in CASES)
    assert any(c[6].get("walks") and c[6].get("split") == 1 for c in CASES)          # results written without sums
