"""The planner of 8-bit products takes each of its kernels for a shape that the parity tests run, and no other for it."""
import os
import subprocess

from linear_i8_shapes import DIRECT, KERNELS, OTHERS, SHAPES
from paper_2406_09425_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_kernel_has_a_shape(tmp_path):
    exe = str(tmp_path / "linear_i8_plan_check")
    subprocess.run([build.hipcc()] + build.COMMON + [os.path.join(ROOT, "tests", "cpp", "linear_i8_plan_check.cpp"), "-o", exe, "-L", build.PKG, "-lsgprs",
                    f"-Wl,-rpath,{build.PKG}"], check=True, capture_output=True)
    asked = [(kernel, *shape, dtype, 256, int(shape[2] % 16 == 0), residual) for kernel, shape in SHAPES for dtype in (0, 1) for residual in (0, 1)]
    r = subprocess.run([exe], input="".join("%d %d %d %d %d %d %d\n" % a[1:] for a in asked), capture_output=True, text=True, check=True)
    plans = [KERNELS[int(line)] for line in r.stdout.split()]
    assert [(a, p) for a, p in zip(asked, plans) if a[0] != p] == [] and len(plans) == len(asked)
    assert set(DIRECT) | set(OTHERS) == set(KERNELS)
    assert all(shape[2] % 16 == 0 for shapes in DIRECT.values() for shape in shapes) and all(shape[2] % 16 for shapes in OTHERS.values() for shape in shapes)
