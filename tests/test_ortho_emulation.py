"""CPU-only checks of what the tests of the updates' products rest on: the emulation comes to the formula, the matrices reach every kernel, and a kernel's mistake
would be far outside the tolerance."""
import os
import subprocess

import pytest
import torch

import nn_experts_reference as ref
import ortho_emulation as emulation
from ortho_sizes import SIZES
from test_gpu_nn_ortho_products import MORE, STEPS, TYPES, both_parts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "ortho_choose.h"
#include <stdio.h>
#include <stdlib.h>
using namespace evg;
// A kernel: both parts or one, which product, its tile, and whether k is shared out; wide or tall where that changes the operands' way through LDS.
static void tell(uint32_t W, uint32_t a, uint32_t b) {
  const uint32_t n = a < b ? a : b, k = a < b ? b : a;
  for (int type = 0; type < 2; ++type)   // bfloat16, others
    for (int op = 0; op < 3; ++op) {
      const bool split = type || n <= 256;
      const OrthoShape s = op == 0 ? OrthoShape{n, n, k, W, 1u << 26} : op == 1 ? OrthoShape{n, n, n, W, 1u << 26} : OrthoShape{a, b, n, W, 1u << 26};
      const OrthoChoice c = choose_ortho(s, op != 2, split);
      printf("%d %d %d %u %d\n", split, op, op == 1 ? 0 : a > b, c.tile, c.parts > 1);
    }
}
int main(int argc, char** argv) {
  if (argc > 1) {
    for (int i = 1; i + 2 < argc; i += 3) tell(atoi(argv[i]), atoi(argv[i + 1]), atoi(argv[i + 2]));
    return 0;
  }
  srand(2);
  for (int i = 0; i < 60000; ++i) {
    auto any = [&](double hi) { return (uint32_t)exp(log(hi) * (rand() / (double)RAND_MAX)); };
    const uint32_t W = rand() % 3 ? 1 : any(65), a = any(16384), b = any(65536);
    if ((double)W * a * b < 1e9) rand() % 2 ? tell(W, a, b) : tell(W, b, a);
  }
}
"""


def test_the_products_tests_run_every_kernel(tmp_path):
    """With at least two steps a test runs the product with X both where it is the last one and where it is not."""
    (tmp_path / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2103_07454_amd", "csrc"), str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)

    def run(*args):
        return {tuple(map(int, line.split())) for line in
                subprocess.run([str(tmp_path / "main"), *map(str, args)], check=True, capture_output=True, text=True).stdout.split("\n") if line}

    tested = {kernel for size in SIZES + MORE for kernel in run(*size)}
    missing = sorted(run() - tested)
    assert not missing, missing
    assert STEPS >= 2 and {both_parts(a, 300, 300) for a, _ in TYPES} == {False, True}


@pytest.mark.parametrize("size", [(1, 1), (3, 5), (20, 30), (64, 64), (130, 65)], ids=lambda s: "x".join(map(str, s)))
def test_emulation_against_the_formula(size):
    """Both parts leave up to 1e-5 of the usual steps' result here, one part 1e-2."""
    u = emulation.gradient(torch.Generator().manual_seed(3), 1, *size)[0]
    want, _ = ref.orthogonal(u.double(), torch.float32, scale=-1.5)
    for both, left in ((True, 1e-5), (False, 1e-2)):
        assert float((emulation.emulate(u, both, None, scale=-1.5) - want).norm()) <= left * float(want.norm())


@pytest.mark.parametrize("types", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("size", [(17, 8), (65, 130), (377, 361), (45, 5912), (899, 1089)], ids=lambda s: "x".join(map(str, s)))
def test_mistakes_are_far_outside_the_tolerance(types, size):
    dtype, out_dtype = types
    u = emulation.gradient(torch.Generator().manual_seed(1), 1, *size)[0].to(dtype).float()
    both = both_parts(dtype, *size)
    want = emulation.emulate(u, both, out_dtype, steps=STEPS)
    room = emulation.tolerance(want, u, both, out_dtype, steps=STEPS)
    off = lambda mistake: float((emulation.emulate(u, both, out_dtype, steps=STEPS, mistake=mistake) - want).norm())  # noqa: E731
    for mistake in ("without gram", "without square", "without apply", "a share of k", "a tile"):
        assert not off(mistake) <= 10 * room, (mistake, off(mistake) / room)
    if out_dtype is torch.float32:      # 16 bits of a result hide what the second part of X is for
        assert off("X in one part") > (20 if both else 1.5) * room
    if dtype is torch.float32 and max(size) < 1000:
        for what in ("gram", "square", "apply"):
            assert off(f"one part, {what}") > 4 * room
