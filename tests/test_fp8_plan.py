"""How aal_fp8_matmul cuts a product, by csrc/aal_fp8_plan.h compiled for the host: the
sizes of the GPU tests reach the kernels that they are there for."""
import os
import shutil
import subprocess

import pytest

import test_gpu_fp8_matmul_scales as scales
import test_gpu_fp8_matmul_tiles as tiles

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

DRIVER = """
#include "aal_fp8_plan.h"
#include <cstdio>
int main() {
  long m, n, k;
  int wide;
  while (scanf("%ld %ld %ld %d", &m, &n, &k, &wide) == 4) {
    const aal::MatmulPlan p = aal::plan_of(m, n, k, wide != 0);
    printf("%d %d\\n", p.kind, p.splits);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    folder = tmp_path_factory.mktemp("plan")
    (folder / "plan.cpp").write_text(DRIVER)
    exe = str(folder / "plan")
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", f"-I{os.path.join(ROOT, 'paper_2609_24150_amd', 'csrc')}",
                    str(folder / "plan.cpp"), "-o", exe], check=True)

    def of(sizes, wide=False):
        r = subprocess.run([exe], input="".join(f"{m} {n} {k} {int(wide)}\n" for m, n, k in sizes), capture_output=True,
                           text=True, check=True)
        return [tuple(map(int, line.split())) for line in r.stdout.splitlines()]

    return of


def test_tiles_of_256(plan):
    assert plan(tiles.SIZES) == [(2, s) for s in tiles.PARTS]
    rows, D, V = 2100, 4100, 2200  # test_gradients_in_bf16
    assert [k for k, _ in plan([(rows, D, V), (V, D, rows)])] == [2, 2]


def test_scales(plan):
    assert [k for k, _ in plan(scales.SIZES)] == [0, 0, 1, 1, 2]
    assert plan(scales.SIZES)[3][1] > 1


def test_fp32_results_take_no_tiles_of_256(plan):
    assert all(k < 2 for k, _ in plan(tiles.SIZES + scales.SIZES, wide=True))


def test_parts_are_not_empty_and_fit(plan):
    """Few rows: at most 32 blocks a part; any cut: every part has a block."""
    sizes = [(m, n, k) for m in (1, 7, 32, 33, 128, 300, 2048) for n in (1, 100, 4000, 33000) for k in (1, 128, 1000, 4097, 70001)]
    for wide in (False, True):
        for (m, n, k), (kind, splits) in zip(sizes, plan(sizes, wide)):
            blocks = -(-k // 128)
            per = -(-blocks // splits)
            assert 1 <= splits <= blocks and (kind != 0 or per <= 32) and (kind == 0) == (m <= 32)
