"""The plans of csrc/mx4_plan.h on the CPU: the sizes of the GPU tests take every tile, whole and split,
and every slab; no plan needs more room than the query says, and the room only grows with the
tokens."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"

PROGRAM = r"""
#include "mx4_plan.h"
#include <cstdio>
#include <cstdlib>
using namespace optima;
int main(int argc, char** argv) {
  for (int i = 1; i + 2 < argc; i += 3) {
    const int64_t n = atoll(argv[i]), d = atoll(argv[i + 1]), ff = atoll(argv[i + 2]);
    const Mx4Plan p = mx4_plan(n, d, ff);
    const Mx4SlabPlan s = mx4_slab_plan(n, d, ff);
    printf("%d %d %d %d %lld %lld %lld\n", p.tile, p.splits, s.tokens, s.splits,
           (long long)mx4_part_bytes(p.tile, p.splits, p.tiles),
           (long long)(s.tokens ? mx4_slab_parts(s.tokens, s.splits, n, ff) : 0),
           (long long)mx4_room(n, d, ff));
  }
}
"""
# Sizes of tests/test_gpu_mx4.py: packed tokens (tile, whether split), and 16-bit ones (tokens of a slab).
TILES = {(4096, 2000, 4096): (0, False), (2000, 14336, 4096): (0, True), (1000, 2000, 4096): (1, False),
         (272, 8192, 3651): (1, True), (400, 2000, 4096): (2, False), (392, 10000, 2897): (2, True),
         (96, 2000, 256): (3, False), (96, 4096, 1000): (3, True), (8, 600, 60000): (2, False),
         (8, 4096, 40000): (3, False)}
SLABS = {(16, 4096, 14336): (16, True), (64, 1000, 14336): (16, False), (9, 14336, 4096): (0, False),
         (64, 200, 20000): (32, False), (17, 4096, 14336): (32, True), (64, 600, 70000): (64, False),
         (33, 14336, 14336): (64, True), (100, 4096, 14336): (32, False), (300, 4096, 4096): (64, True),
         (96, 4096, 4096): (32, True)}


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
def test_sizes_take_every_tile(plans):
    assert {s: (p[0], p[1] > 1) for s, p in zip(TILES, plans(TILES))} == TILES
    assert set(TILES.values()) == {(t, split) for t in range(4) for split in (False, True)}


@pytest.mark.slow
def test_sizes_take_every_slab(plans):
    assert {s: (p[2], p[3] > 1) for s, p in zip(SLABS, plans(SLABS))} == SLABS


@pytest.mark.slow
def test_room(plans):
    for d, ff in ((64, 64), (512, 5000), (1001, 2731), (4096, 4096), (14336, 4096), (14336, 14336),
                  (4096, 128000), (1 << 20, 64), (100, 1 << 24), (1 << 20, 20000)):
        last = 0
        for n, p in ((n, plans([(n, d, ff)])[0]) for n in (
                1, 2, 8, 9, 15, 16, 17, 32, 33, 63, 64, 65, 100, 129, 257, 513, 777, 1024, 2000, 4096, 10000,
                100000, 1 << 21)):
            assert p[6] >= last and p[6] >= p[4] and p[6] >= p[5] and (n > 8 or p[6] == 0)
            last = p[6]
