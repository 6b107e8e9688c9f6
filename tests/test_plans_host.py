"""The plans of csrc/gated_plan.h on the CPU: the sizes of the GPU tests take the kernels, tiles and
splits that they are there for, whatever the constants become."""
import os
import shutil
import subprocess

import pytest

from test_gpu_gated_plans import FEW, GRADIENTS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"

PROGRAM = r"""
#include "gated_plan.h"
#include <cstdio>
#include <cstdlib>
int main(int argc, char** argv) {
  for (int i = 1; i + 2 < argc; i += 3) {
    const int64_t n = atoll(argv[i]), d = atoll(argv[i + 1]), ff = atoll(argv[i + 2]);
    const optima::GradPlan p = optima::plan_grad(n, d, ff);
    const optima::GatedPlan f = optima::plan_gated(n, d, ff);
    printf("%d %d %d %d %d %d\n", p.side, p.splits[0], p.splits[1],
           int(optima::few_tokens(n, d, ff)), int(f.wide), f.splits);
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc is not installed")
    at = tmp_path_factory.mktemp("plans")
    src, obj, exe = (str(at / n) for n in ("t.hip", "t.o", "t"))
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([HIPCC, "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-O1", "-fPIC",
                    "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2512_13886_amd", "csrc"), "-c", src, "-o", obj],
                   check=True, timeout=300)
    subprocess.run(["g++", obj, "-o", exe], check=True, timeout=120)

    def run(sizes):
        r = subprocess.run([exe, *(str(v) for s in sizes for v in s)], capture_output=True, text=True,
                           check=True, timeout=60)
        return [tuple(int(v) for v in line.split()) for line in r.stdout.splitlines()]
    return run


@pytest.mark.slow
def test_gradients_take_both_tiles_split_and_whole(plans):
    got = plans(GRADIENTS)
    assert [p[:3] for p in got] == list(GRADIENTS.values())
    large = [p for p in got if p[0] == 256]
    assert any(p[1:3] == (1, 1) for p in large)
    assert any(p[1] > 1 for p in large) and any(p[2] > 1 for p in large)
    # The layer of the headline figures.
    assert plans([(4096, 4096, 14336)])[0][0] == 256


@pytest.mark.slow
def test_few_tokens_are_streamed(plans):
    assert all(p[3] for p in plans(FEW))
    assert plans([(1, 4096, 14336)])[0][3]


@pytest.mark.slow
def test_forward_takes_both_tiles_and_splits(plans):
    # Of tests/test_gpu_gated.py: large tiles, both, split sums.
    large, both, split = plans([(4096, 128, 2048), (700, 960, 12529), (300, 1000, 33)])
    assert large[4] == 2048 and 0 < both[4] < 12529 and split[4] == 0 and split[5] > 1
