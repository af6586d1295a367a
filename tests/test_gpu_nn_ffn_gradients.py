"""The block's backward pass where not all gradients are wanted: weights that are held fixed cost nothing."""
import itertools

import pytest
import torch

from test_gpu_nn_ffn import NAMES, check, tensors, train

pytestmark = pytest.mark.gpu
DW = NAMES[2:]


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


@pytest.mark.parametrize("size", [(2, 30, 64, 72), (1, 130, 72, 90)], ids=str)
def test_any_of_the_weights_gradients(nn, size):
    t = tensors(*size, torch.bfloat16, seed=20)
    op, want = train(nn, t, torch.bfloat16, "silu")
    args = (t["x"], t["w_gate"], t["w_up"], t["w_down"])
    _, saved = op.forward(*args, save=True)
    for some in itertools.product((False, True), repeat=3):
        given = {k: torch.full_like(want[k], 7.0) for k, s in zip(DW, some) if s}
        got = op.backward(t["dy"], *args, saved, weight_gradients=False, **given)
        for k, g in zip(NAMES[1:], got):
            if k == "dx" or k in given:
                assert torch.equal(g, want[k]), k
                assert k == "dx" or g is given[k]
            else:
                assert g is None
    assert op.backward(t["dy"], *args, saved, input_gradient=False, weight_gradients=False) == (None, None, None, None)
    check("silu", torch.bfloat16, t, want, NAMES)
