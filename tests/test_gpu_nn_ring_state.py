"""FFNRing's forward pass by itself: it answers with the ring's present parameters, whatever type it computes in."""
import pytest
import torch

from test_gpu_nn_ring import data

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
def test_forward_answers_with_the_present_parameters(dtype):
    from paper_2103_07454_amd import ffn_ring
    run = ffn_ring.FFNRing(3, width=64, hidden=96, tokens=20, dtype=dtype, lr=0.5, max_norm=10.0)
    x, target = data(run, 0)

    def expected():
        fresh = ffn_ring.FFNRing(3, width=64, hidden=96, tokens=20, dtype=dtype)
        fresh.ring.x.copy_(run.ring.x)
        fresh.low.copy_(fresh.ring.x)
        return fresh.forward(x)[0]

    assert torch.equal(run.forward(x)[0], expected())          # ahead of the first step
    before = run.forward(x)[0]
    for k in range(3):
        run.step(x, target)
    after = run.forward(x)[0]
    assert torch.equal(after, expected()) and not torch.equal(after, before)
