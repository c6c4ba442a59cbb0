"""Failures of the device under ff_adamw_set_create, on the CPU (tests/sanitize/set_create.cpp): status, handle, memory, and
that no error of the runtime is left for the next launch to report as its own."""
import os
import shutil
import subprocess

import pytest

pytest.importorskip("torch")
from paper_2608_26430_amd import binding  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_a_failed_creation_leaves_nothing_behind(tmp_path):
    lib = binding.library_path()
    exe = str(tmp_path / "set_create")
    # (-rdynamic: the program's functions stand before the runtime's for the library too)
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "sanitize", "set_create.cpp"), lib,
                    "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath," + os.path.dirname(lib), "-Wl,-rpath,/opt/rocm/lib",
                    "-Wl,--allow-shlib-undefined", "-o", exe], check=True, timeout=300)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "set creation: 0 failed checks" in run.stdout, run.stdout + run.stderr
