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
    const Mx4FewPlan f = mx4_few_plan(n, d, ff, false);
    printf("%d %d %d %d %d\n", int(mx4_packed_tiles(n, ff, true)), int(mx4_packed_tiles(n, ff, false)),
           mx4_slab_plan(n, d, ff).tokens, f.blocks, f.waves);
  }
}
"""
# Sizes of tests/test_gpu_mx4.py's kind for few 16-bit tokens, that slabs do not take: (blocks of 16 outputs,
# waves). Widths that are no multiple of 8 take the kernel's ragged form, in four tokens at a time.
FEW = {(1, 4097, 5001): (1, 9), (1, 4096, 5000): (1, 8), (3, 1001, 66000): (2, 2), (4, 1000, 66000): (2, 2),
       (2, 14337, 66001): (2, 8), (8, 4097, 14336): (2, 8), (6, 1001, 13000): (2, 2), (5, 1000, 13000): (2, 2),
       (7, 4097, 5001): (1, 8), (9, 1001, 9000): (2, 2), (16, 1001, 9000): (2, 2), (12, 1000, 9000): (2, 2),
       (9, 14335, 4000): (1, 16), (16, 8191, 4000): (1, 9), (10, 8192, 4000): (1, 15),
       (1, 7, 70000): (1, 1), (4, 7, 70000): (2, 1), (8, 5, 13000): (2, 1)}


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


@pytest.mark.slow
def test_sizes_take_every_few_token_form(plans):
    got = plans(FEW)
    assert all(p[2] == 0 for p in got), [s for s, p in zip(FEW, got) if p[2]]
    assert {s: (p[3], p[4]) for s, p in zip(FEW, got)} == FEW
    # Up to 4 tokens and more, one block and two, widths of multiples of 8 and others.
    assert {(n > 4, b, d % 8 > 0) for (n, d, _), (b, _) in FEW.items()} == {
        (a, b, c) for a in (False, True) for b in (1, 2) for c in (False, True)}
