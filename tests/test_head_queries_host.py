"""What the query of a head says of its calls, without a GPU: launches with and without a mask (tests/host/head_masks.cpp), and the products that backward makes."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2304_07741_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_launches_with_a_mask(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    B.load()
    libdir = os.path.dirname(B.LIB_PATH)
    exe = str(tmp_path / "head_masks")
    subprocess.run(["g++", "-O2", "-std=c++17", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "host", "head_masks.cpp"),
                    "-o", exe, f"-L{libdir}", "-lcanvas_dag", f"-Wl,-rpath,{libdir}", "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"], check=True)
    p = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    m = re.search(r"^calls (\d+) wrong (\d+) several (\d+)$", p.stdout, re.M)
    assert m and p.returncode == 0 and int(m[2]) == 0, p.stdout[-4000:] + p.stderr[-1000:]
    assert int(m[1]) > 900 and int(m[3]) > 5


@pytest.mark.parametrize("rows,features,classes,dtype,again", [
    (4, 2048, 131072, B.CANVAS_BF16, 0),             # few rows: forward leaves their logits
    (256, 512, 1000, B.CANVAS_F32, 0),
    (4096, 4096, 32768, B.CANVAS_BF16, 0),           # all pieces' logits are left
    (4096, 1024, 32768, B.CANVAS_BF16, 1),           # none
    (1000, 64, 5000, B.CANVAS_BF16, 1)])
def test_products_of_backward(rows, features, classes, dtype, again):
    h = B.canvas_head_compile(rows, features, classes, dtype)
    info = B.canvas_head_query(h)
    assert info.flops_fwd == 2.0 * rows * features * classes and info.flops_bwd == (2 + again) * info.flops_fwd
    B.canvas_head_destroy(h)


def test_products_of_some_pieces_are_made_again():
    h = B.canvas_head_compile(24000, 2056, 12000, B.CANVAS_BF16)
    info = B.canvas_head_query(h)
    first = 6144                                       # classes of the first of two pieces
    assert info.pieces == 2 and info.flops_bwd == 2.0 * 24000 * 2056 * (2 * 12000 + 12000 - first)
    B.canvas_head_destroy(h)
