"""The choice of tiles for the products of orthogonal updates, on the CPU: what the tests on the GPU run is all that calls can reach."""
import os
import subprocess
import sys

import pytest

from ortho_sizes import SIZES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "ortho_choose.h"
#include <stdio.h>
#include <stdlib.h>
using namespace evg;
static void tell(uint32_t W, uint32_t a, uint32_t b) {
  const uint32_t n = a < b ? a : b, k = a < b ? b : a;
  for (int split = 0; split < 2; ++split)
    for (int op = 0; op < 3; ++op) {
      const OrthoShape s = op == 0 ? OrthoShape{n, n, k, W, 1u << 26} : op == 1 ? OrthoShape{n, n, n, W, 1u << 26} : OrthoShape{a, b, n, W, 1u << 26};
      const OrthoChoice c = choose_ortho(s, op != 2, split);
      const uint32_t steps = (s.K + (split ? 31 : 63)) / (split ? 32 : 64);
      const bool fits = ortho_partial(s, op != 2, c) <= s.room && c.parts >= 1 && c.parts <= 8 && c.parts <= steps;
      printf("%d %d %u %d %d\n", split, op, c.tile, c.parts > 1, fits);
    }
}
int main(int argc, char** argv) {
  if (argc > 1) {
    for (int i = 1; i + 2 < argc; i += 3) tell(atoi(argv[i]), atoi(argv[i + 1]), atoi(argv[i + 2]));
    return 0;
  }
  srand(1);
  for (int i = 0; i < 60000; ++i) {
    auto any = [&](double hi) { return (uint32_t)exp(log(hi) * (rand() / (double)RAND_MAX)); };
    const uint32_t W = rand() % 3 ? 1 : any(65), a = any(16384), b = any(65536);
    if ((double)W * a * b < 1e9) rand() % 2 ? tell(W, a, b) : tell(W, b, a);
  }
}
"""


@pytest.fixture(scope="module")
def reached(tmp_path_factory):
    where = tmp_path_factory.mktemp("ortho")
    (where / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2103_07454_amd", "csrc"), str(where / "main.cpp"), "-o", str(where / "main")], check=True)

    def run(*args):
        lines = subprocess.run([str(where / "main"), *map(str, args)], check=True, capture_output=True, text=True).stdout.split("\n")
        rows = [tuple(map(int, line.split())) for line in lines if line]
        assert all(r[-1] for r in rows), "partial sums that do not fit, or parts without a step"
        return {r[:-1] for r in rows}

    return run


def test_the_tests_run_every_kernel_that_calls_reach(reached):
    any_call, tested = reached(), reached(*[v for s in SIZES for v in s])
    print(sorted(any_call - tested), file=sys.stderr)
    assert any_call <= tested


def test_tiles_of_256_are_of_one_part_of_each_operand(reached):
    """The kernels that there are: no others may be asked for."""
    for split, op, tile, parts in reached():
        assert tile in (64, 128, 256) and not (tile == 256 and (split or (op == 2 and parts)))
