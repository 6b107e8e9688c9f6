"""Which kernel takes few tokens and odd scales (csrc/mx4_plan.h), on the CPU."""
import os
import subprocess

import pytest

from test_mx4_plans_host import HIPCC, ROOT

PROGRAM = r"""
#include "mx4_plan.h"
#include <cstdio>
#include <cstdlib>
using namespace optima;
int main(int argc, char** argv) {
  for (int i = 1; i + 2 < argc; i += 3) {
    const int64_t n = atoll(argv[i]), d = atoll(argv[i + 1]), ff = atoll(argv[i + 2]);
    printf("%d %d\n", int(mx4_packed_tiles(n, ff, true)), int(mx4_packed_tiles(n, ff, false)));
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
def test_odd_scales_never_take_tiles(plans):
    """The tiles' direct loads of scales are 16 bytes at multiples of 16."""
    sizes = [(n, 4096, ff) for n in (1, 8, 9, 16, 17, 64, 600, 1 << 21) for ff in (64, 9000, 128000)]
    assert all(p[1] == 0 for p in plans(sizes))
    assert [p[0] for p in plans([(16, 4096, 4096), (16, 4096, 9000), (8, 8192, 28672), (17, 64, 64)])] == [
        0, 1, 0, 1]
