"""The gated feed-forward block through every kernel that its calls can launch, against its definition in 64 bits (bounds:
tests/nn_reference.py).  That these cases and test_gpu_nn_ffn.SIZES leave none out is tests/test_ffn_choose.py's to check."""
import pytest
import torch

from test_gpu_nn_ffn import NAMES, SHORT, TYPES, check, tensors, train

pytestmark = pytest.mark.gpu

#: (workers, tokens, width, hidden), activation, whether the tensors begin one element beyond a 16-byte unit.
CASES = [((1, 13, 624, 72), "gelu", False), ((1, 33, 69, 70), "gelu", False), ((1, 693, 152, 424), "gelu", False),
         ((1, 1085, 740, 392), "gelu", False), ((3, 1, 2240, 822), "gelu", False), ((3, 2302, 79, 977), "gelu", False),
         ((3, 2368, 1032, 72), "gelu", False), ((1, 2405, 64, 2647), "silu", False), ((1, 4385, 64, 664), "silu", False),
         ((2, 37, 1032, 4632), "silu", False), ((3, 1749, 1142, 64), "silu", False), ((1, 17, 64, 72), "gelu", True),
         ((1, 86, 400, 64), "gelu", True), ((1, 589, 296, 232), "gelu", True), ((2, 135, 711, 424), "gelu", True),
         ((2, 358, 76, 4431), "gelu", True), ((1, 71, 72, 64), "silu", True), ((1, 139, 760, 800), "silu", True)]


def beyond_a_unit(t):
    flat = torch.full((t.numel() + 1,), float("nan"), dtype=t.dtype, device=t.device)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("size,kind,misaligned", CASES, ids=str)
def test_every_kernel(nn, dtype, size, kind, misaligned):
    t = tensors(*size, dtype, seed=sum(size))
    if misaligned:
        t = {k: beyond_a_unit(v) for k, v in t.items()}
    _, got = train(nn, t, dtype, kind)
    check(kind, dtype, t, got, NAMES, device="cuda")
