"""The order of what an attention call over an 8-bit cache or of drafted trees enqueues (tests/step_order.cpp)."""
import os
import shutil
import subprocess

import pytest

from paper_2505_03756_amd import flpool

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_order_waits_and_refusals(tmp_path):
    """The workspace of cut contexts is waited for across streams, records are uploaded before they are read, and a call that finds no memory
    has enqueued nothing."""
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    flpool.load()
    pkg, exe = os.path.join(ROOT, "paper_2505_03756_amd"), str(tmp_path / "step_order")
    b = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(ROOT, "include"),
                        "-I" + os.path.join(pkg, "csrc"), "-I/opt/rocm/include", os.path.join(ROOT, "tests", "step_order.cpp"),
                        "-rdynamic", flpool.LIB_PATH, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib:" + pkg, "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert b.returncode == 0, b.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "in order" in r.stdout, (r.stdout + r.stderr)[-3000:]
