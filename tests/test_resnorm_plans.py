"""The launches of the join's sums (csrc/resnorm_plan.h, compiled and asked on the CPU)."""
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
