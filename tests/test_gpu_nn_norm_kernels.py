"""Every kernel of the norms: each number of threads to a row, both norms, all types, with and without a gate and a norm behind the block."""
import itertools

import pytest

from test_gpu_nn_blocknorm import SHORT, TYPES, check, tensors

pytestmark = pytest.mark.gpu

#: Widths in eights take kernels for which gate and norm are known; their odd neighbours one that asks at run time.
WIDTHS = [120, 248, 504, 1000, 2040, 4088, 8184, 8208]


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("width", WIDTHS)
def test_every_kernel(nn, dtype, kind, width):
    for D, gate, post in itertools.product((width, width + 3), (0, 2), (False, True)):
        t, d_out, d_normed = tensors(2, 5, D, dtype, kind, gate, post=post, seed=D)
        check(nn, kind, dtype, t, d_out, d_normed, gate)
