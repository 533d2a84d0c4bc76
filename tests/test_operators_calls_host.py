"""What the entry points of the operators around a block hand to the runtime, and what they refuse: a program that has the runtime's launch
functions itself (tests/host/operator_calls.cpp), so that nothing reaches a GPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2304_07741_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    B.load()
    libdir = os.path.dirname(B.LIB_PATH)
    exe = str(tmp_path_factory.mktemp("calls") / "operator_calls")
    subprocess.run(["g++", "-O2", "-std=c++17", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "host", "operator_calls.cpp"),
                    "-o", exe, f"-L{libdir}", "-lcanvas_dag", f"-Wl,-rpath,{libdir}", "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"], check=True)
    return exe


def _look(program, what):
    p = subprocess.run([program, what], capture_output=True, text=True, timeout=300)
    m = re.search(rf"^{what} cases (\d+) wrong (\d+)$", p.stdout, re.M)
    assert m and p.returncode == 0 and int(m[2]) == 0, p.stdout[-4000:] + p.stderr[-1000:]
    return int(m[1])


def test_tensors_that_share_bytes_are_refused(program):
    assert _look(program, "overlap") > 5000


def test_lds_is_asked_for_whatever_shapes_came_before(program):
    assert _look(program, "lds") > 200


def test_no_launch_has_too_many_threads(program):
    assert _look(program, "threads") > 1000
