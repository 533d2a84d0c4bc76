"""Rows of any length taken in pieces of eight elements, on the CPU: nothing behind a tensor's end is read (tests/host/row_pieces.cpp)."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_nothing_behind_the_end_is_read(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "row_pieces")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wno-unknown-pragmas", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    os.path.join(ROOT, "tests", "host", "row_pieces.cpp"), "-o", exe], check=True)
    p = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    m = re.search(r"^pieces (\d+) wrong (\d+)$", p.stdout, re.M)
    assert p.returncode == 0 and m and int(m[1]) > 100000 and int(m[2]) == 0, (p.returncode, p.stdout, p.stderr)
