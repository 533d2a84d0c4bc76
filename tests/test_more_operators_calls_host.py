"""What the entry points of gated pairs, heads and the clipping of gradients hand to the runtime: a program that has the runtime's launch functions
itself (tests/host/more_operator_calls.cpp), so that nothing reaches a GPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2304_07741_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_launches_are_what_the_plans_say(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    B.load()
    libdir = os.path.dirname(B.LIB_PATH)
    exe = str(tmp_path / "more_operator_calls")
    subprocess.run(["g++", "-O2", "-std=c++17", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "host", "more_operator_calls.cpp"),
                    "-o", exe, f"-L{libdir}", "-lcanvas_dag", f"-Wl,-rpath,{libdir}", "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"], check=True)
    p = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    m = re.search(r"^launches cases (\d+) wrong (\d+)$", p.stdout, re.M)
    assert m and p.returncode == 0 and int(m[2]) == 0, p.stdout[-4000:] + p.stderr[-1000:]
    assert int(m[1]) > 3000
