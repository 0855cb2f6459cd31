"""The shapes of the GPU tests reach every kernel of the 8-bit product, with rows
at 16-byte boundaries and without: asked from the library's own rule, on the
host, so that a moved threshold cannot leave a kernel untested."""
import os
import shutil
import subprocess

import pytest

from product_shapes import ALIGNED, RAGGED

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNELS = 7   # enum QLinearKernel: five tiles, two direct ones


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("plan") / "qlinear_plan_check")
    res = subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", f"-I{os.path.join(ROOT, 'paper_2412_00119_amd', 'csrc')}",
                          os.path.join(ROOT, "tests", "qlinear_plan_check.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr

    def ask(shapes):
        text = "".join(f"{n} {m} {k + pad} {k} {lead}\n" for n, m, k, pad, lead in shapes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=60, check=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return ask


def test_every_kernel_is_reached(plan):
    aligned, ragged = plan(ALIGNED), plan(RAGGED)
    assert all(r == 0 for _, r in aligned) and all(r == 1 for _, r in ragged)
    assert {k for k, _ in aligned} == set(range(KERNELS))
    assert {k for k, _ in ragged} == set(range(KERNELS))


def test_the_rule_at_its_edges(plan):
    """One row more or fewer, the 8192 outputs, and rows too far apart for a tile."""
    far = (1 << 21) + 1
    got = [k for k, _ in plan([(16, 8191, 64, 0, 0), (16, 8192, 64, 0, 0), (17, 100, 64, 0, 0), (32, 100, 64, 0, 0),
                               (33, 100, 64, 0, 0), (33, 100, 64, far - 64, 0), (33, 100, 64, far - 65, 0),
                               (8192, 8192, 64, 0, 0), (1 << 20, 2 ** 31 - 1, 1, 0, 0), (1, 2 ** 31 - 1, 1, 0, 0)])]
    assert got == [5, 6, 6, 6, 4, 6, 4, 0, 0, 6]
