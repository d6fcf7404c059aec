"""How many clusters run at a time is kept by device and share (CPU only: the header that the launch takes it from, compiled
by itself)."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_11185_gb300", "csrc")


def test_answers_of_devices_and_shares_stay_apart(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path / "cluster_counts")
    r = subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-I", CSRC,
                        os.path.join(ROOT, "tests", "c_abi", "cluster_counts.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert subprocess.run([exe], timeout=60).returncode == 0


def test_the_launch_asks_for_the_current_device():
    with open(os.path.join(CSRC, "distill.cu")) as f:
        src = f.read()
    body = src[src.index("cudaError_t launch_held("):src.index("cudaError_t launch_block(")]
    assert re.search(r"cudaGetDevice\(&(\w+)\)", body) and re.search(r"\.find\(device, ", body)
    assert body.index("cudaGetDevice") < body.index(".find(") < body.index("cudaOccupancyMaxActiveClusters") < body.index(".keep(")
