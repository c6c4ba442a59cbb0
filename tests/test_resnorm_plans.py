"""Which instances of the join's kernels the sizes of the GPU tests run, and the launches of its sums (csrc/resnorm_plan.h, compiled and
asked on the CPU)."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("plans") / "resnorm_plans")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I" + os.path.join(ROOT, "paper_2608_26430_amd", "csrc"),
                    os.path.join(HERE, "plans", "resnorm_plans.cpp"), "-o", exe], check=True, timeout=300)

    def lines(questions):
        out = subprocess.run([exe], input="\n".join(questions) + "\n", capture_output=True, text=True, check=True, timeout=120).stdout
        return [[int(x) for x in line.split()] for line in out.splitlines()]

    return lines


@pytest.mark.parametrize("n", [1, 31, 33, 4096, 1 << 20, (1 << 24) - 31, 1 << 24])
@pytest.mark.parametrize("vectors", [0, 1, 4])
def test_launches_of_the_sums_have_fewer_than_two_to_the_32_threads(ask, n, vectors):
    for groups in (1, 3, 4, 7, 100, 511):
        row, = ask([f"sums {n} {vectors} {groups}"])
        threads, rows = row[::2], row[1::2]
        assert all(0 < t < 2 ** 32 for t in threads) and all(r > 0 for r in rows) and sum(rows) == groups, (groups, row)


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("esz", [2, 4])
def test_sizes_run_every_instance(ask, esz, backward):
    pytest.importorskip("torch")
    from tests.test_gpu_resnorm_instances import KINDS, SIZES
    widths = sorted({n + d for n in [1, 4, 8, 9000, 20000] + [1 << k for k in range(4, 15)] for d in range(-9, 10) if n + d > 0} | set(range(3, 9000, 97)))
    every = [(T, n) for T in (1, 512, 513, 100_000) for n in widths]
    shapes = {tuple(s) for s in ask([f"shape {T} {n} {esz} {backward}" for T, n in every]) if s[1]}
    run = {tuple(s) for s in ask([f"shape {T} {n} {esz} {backward}" for T, n in SIZES]) if s[1]}
    assert run == shapes, (shapes - run, run - shapes)
    # rows that are read several times, too
    assert any(not s[1] for s in ask([f"shape {T} {n} {esz} {backward}" for T, n in SIZES]))
    # the backward's groups of instances: norms on both sides, after, before, none, each as RMS without biases and otherwise
    assert {(post != "none", norm != "none", bias or "layer" in (post, norm)) for post, norm, bias in KINDS} == {
        (True, True, False), (True, True, True), (False, True, False), (False, True, True), (True, False, True), (False, False, False)}
