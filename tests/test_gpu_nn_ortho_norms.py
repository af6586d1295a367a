"""Orthogonal updates of matrices whose norm is near the ends of what 32 bits hold."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("power", [-133, -126, -119, -110, -60, 60, 115])
@pytest.mark.parametrize("momentum", [False, True], ids=["gradient", "momentum"])
def test_a_power_of_two_changes_nothing_without_eps(nn, dtype, power, momentum):
    """Elements of three bits, so that those of the scaled matrix are exact even where they are subnormal: norm, quotient and product are scaled alike, and every
    bit of the update is the same.  With a norm below 2^14 / 2^128 the factor that takes it to 1 has no value in 32 bits."""
    gen = torch.Generator(device="cuda").manual_seed(power + 200)
    grad = torch.randint(-7, 8, (2, 40, 72), generator=gen, device="cuda").to(dtype)
    old = torch.randint(-7, 8, (2, 40, 72), generator=gen, device="cuda").float()
    small = (grad.double() * 2.0 ** power).to(dtype)
    assert torch.equal(small.double(), grad.double() * 2.0 ** power)
    op = nn.Orthogonal(40, 72, matrices=2, dtype=dtype, eps=0.0, momentum=0.5)
    want = op.update(grad, momentum=old.clone() if momentum else None)
    m = (old.double() * 2.0 ** power).float() if momentum else None
    got = op.update(small, momentum=m)
    assert torch.isfinite(want).all() and float(want.abs().max()) > 0.0
    assert torch.equal(got, want)


def test_one_element(nn):
    """The smallest subnormal and the largest number, alone in their matrices."""
    for value in (2.0 ** -149, 2.0 ** -126, 1.0, torch.finfo(torch.float32).max):
        grad = torch.zeros(1, 3, 5, device="cuda")
        grad[0, 1, 2] = value
        out = nn.Orthogonal(3, 5, eps=0.0, steps=1, polynomial=(1.0, 0.0, 0.0)).update(grad)
        assert abs(float(out[0, 1, 2]) - 1.0) <= 2.0 ** -20 and int((out != 0).sum()) == 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("power", [-80, -70, -30, 30, 100])
@pytest.mark.parametrize("polynomial", [(3.4445, -4.7750, 2.0315), (1.0, 0.0, 0.0)], ids=["usual", "none"])
def test_a_scale_that_is_a_power_of_two_is_exact(nn, dtype, power, polynomial):
    """Down to the smallest scale that is taken: what it is multiplied with on the way keeps all bits.  Updates of 16 significant bits or more stay normal numbers."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    grad = torch.randn(1, 40, 300, generator=gen, device="cuda").to(dtype)
    make = lambda scale: nn.Orthogonal(40, 300, dtype=dtype, polynomial=polynomial, scale=scale).update(grad)  # noqa: E731
    assert torch.equal(make(2.0 ** power).double(), make(1.0).double() * 2.0 ** power)
    assert float(make(0.0).abs().max()) == 0.0
