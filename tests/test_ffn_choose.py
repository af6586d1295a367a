"""The choice of tiles on the CPU: every kernel that a block of the operators' range can launch has a test that runs it."""
import random

import pytest

import ffn_dispatch
from perf import operators

TYPES = ("bf16", "f16", "f32")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return ffn_dispatch.compile_chooser(str(tmp_path_factory.mktemp("choose")))


def of(case):
    return tuple(case[k] for k in ("workers", "tokens", "width", "hidden", "dtype", "activation", "train"))


def test_every_kernel_that_calls_reach_is_tested(exe):
    import test_gpu_nn_ffn
    import test_gpu_nn_ffn_tiles
    rng = random.Random(0)
    drawn = [operators.draw(rng) for _ in range(12_000)] + operators.listed()
    calls = [of(c) for c in drawn if c["op"] == "ffn"]
    reached = set().union(*ffn_dispatch.kernels(exe, calls + [(*c, True) for c in calls]))
    tested = [(*size, t, "silu", True) for size in test_gpu_nn_ffn.SIZES for t in TYPES]
    tested += [(*size, t, kind, True, misaligned) for size, kind, misaligned in test_gpu_nn_ffn_tiles.CASES for t in TYPES]
    missing = reached - set().union(*ffn_dispatch.kernels(exe, tested))
    assert len(reached) > 150 and not missing, sorted(missing, key=str)


@pytest.mark.parametrize("case,want", [
    ((1, 1, 2048, 5632, "bf16", "silu", False), {("bf16", "gated", False, "rows", 8), ("bf16", "down", False, "rows", 8)}),
    ((1, 8192, 2048, 8192, "bf16", "silu", True), {("bf16", "gated", False, "256", True), ("bf16", "down", False, "256", True),
                                                   ("bf16", "gated_bwd", False, "128", True), ("bf16", "input", False, "256", True),
                                                   ("bf16", "weight", False, "256", True)})])
def test_measured_cases(exe, case, want):
    assert ffn_dispatch.kernels(exe, [case])[0] == want
