"""The rotation's table of angles in shared memory: what a launch asks for holds what its kernel reaches, for every
rotated size (CPU only: the header that both take it from, compiled by itself)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_table_holds_every_entry(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path / "rope_table")
    r = subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2607_11185_gb300", "csrc"),
                        os.path.join(ROOT, "tests", "c_abi", "rope_table.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout[-200:])
    lines = [tuple(map(int, x.split())) for x in r.stdout.splitlines()]
    assert [x[:3] for x in lines] == [(rot, i, c) for rot in range(16, 257, 16) for i in (0, 1) for c in range(1, 9)]
    for rot, inter, copies, asked, reached in lines:
        assert rot // 2 * copies * 4 * 8 <= reached <= asked <= 48 * 1024, (rot, inter, copies, asked, reached)
