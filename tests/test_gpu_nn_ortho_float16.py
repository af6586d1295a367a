"""Updates of float16 gradients are as exact as their type: what the steps leave is below the rounding of the result, at every size and spectrum."""
import pytest
import torch

import nn_experts_reference as ref
import ortho_emulation as emulation

pytestmark = pytest.mark.gpu

SIZES = [(4, 4), (16, 16), (16, 60), (64, 64), (128, 784), (256, 256), (700, 512), (512, 1365)]


def directions(gen, kind, rows, cols):
    make = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    if kind == "all alike":
        return make(rows, cols)
    few = max(1, min(rows, cols) // 16)
    strong = make(rows, few) @ make(few, cols) / few ** 0.5
    return strong if kind == "few" else strong + 0.1 * make(rows, cols)


@pytest.mark.parametrize("kind", ["all alike", "few", "few strong"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_five_steps(size, kind):
    """Against the same arithmetic, and against the formula: the kernel may be off by the rounding of the result, what the parts leave and what sums in 32 bits do."""
    from paper_2103_07454_amd import nn
    gen = torch.Generator().manual_seed(sum(size))
    for _ in range(3):
        grad = directions(gen, kind, *size).half()
        u = grad.float()
        wide = nn.Orthogonal(*size, dtype=torch.float16, out_dtype=torch.float32).update(grad.cuda()[None])[0].double().cpu()
        want = emulation.emulate(u, True, torch.float32)
        room = emulation.tolerance(want, u, True, torch.float32)
        off = float((wide - want).norm())
        assert off <= room, (off / float(want.norm()), room / float(want.norm()))
        exact, _ = ref.orthogonal(u.double(), torch.float32)
        half = nn.Orthogonal(*size, dtype=torch.float16).update(grad.cuda()[None])[0].double().cpu()
        rounding = float((exact.half().double() - exact).norm())
        left = float((want - exact).norm()) + room
        off = float((half - exact).norm())
        print(f"[ortho f16] {size} {kind}: off by {off / float(exact.norm()):.2e} of the update, its rounding {rounding / float(exact.norm()):.2e}, parts and sums at most {left / float(exact.norm()):.1e}", flush=True)
        # where what is left moves a value across the border between two float16, that adds at most as much as is left
        assert off <= rounding + 2 * left
        # What the parts leave, of the emulation alone: `room` is four times a bound of what any sums in 32 bits do, which a few directions' rounding error, stretched 485-fold, makes
        # as large as the rounding itself, and says nothing of the parts.
        assert float((want - exact).norm()) <= 0.5 * rounding
