"""Ring workers that train in 16 bits of which few are exponents: the loss's scale keeps their gradients above the subnormals."""
import pytest
import torch

import nn_reference as ref
from test_gpu_nn_ring import data, reference_gradient

pytestmark = pytest.mark.gpu


def test_gradients_of_many_values():
    """A million values a worker: the gradient of each value of the output is some 1e-7 of it."""
    from paper_2103_07454_amd import ffn_ring
    run = ffn_ring.FFNRing(3, blocks=1, width=1024, hidden=64, tokens=1024, dtype=torch.float16, max_norm=0.05)
    x, target = data(run, 3)
    run.low.copy_(run.ring.x)
    want, norms = reference_gradient(run, x, target)
    _, norm = run.step(x, target)
    got = torch.from_numpy(run.ring.layout.unpad(run.grad.cpu().numpy())).double()
    off = (got - want).norm(dim=1) / want.norm(dim=1)
    print(f"[ring] f16: gradients off by {off.max() / ref.UNIT[torch.float16]:.2f} units", flush=True)
    # as for few values: some ten roundings on the way, and as much again through the norms
    assert float(off.max()) <= 20 * ref.UNIT[torch.float16]
    assert all(abs(a / b - 1) <= 20 * ref.UNIT[torch.float16] for a, b in zip(norm.tolist(), norms))


def test_training_lowers_the_loss():
    from paper_2103_07454_amd import ffn_ring
    run = ffn_ring.FFNRing(4, width=64, hidden=192, blocks=2, tokens=1500, dtype=torch.float16, lr=0.2, max_norm=1.0)
    losses = []
    for k in range(40):
        loss, norm = run.step(*data(run, k))
        assert torch.isfinite(norm).all()
        losses.append(float(loss.mean()))
    print(f"[ring] f16 loss {losses[0]:.4f} -> {losses[-1]:.4f}", flush=True)
    assert losses[-1] < 0.7 * losses[0]


def test_a_gradient_that_overflows_sits_the_step_out():
    from paper_2103_07454_amd import ffn_ring
    run = ffn_ring.FFNRing(3, width=64, hidden=96, tokens=30, dtype=torch.float16, loss_scale=2.0 ** 60)
    before = run.ring.state("x")
    loss, norm = run.step(*data(run, 0))
    assert torch.isfinite(loss).all() and not torch.isfinite(norm).any()
    assert float(run.grad.abs().max()) == 0.0 and (run.ring.state("x") == before).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_other_types_are_not_scaled(dtype):
    from paper_2103_07454_amd import ffn_ring
    assert ffn_ring.FFNRing(3, width=64, hidden=96, tokens=30, dtype=dtype).loss_scale == 1.0
