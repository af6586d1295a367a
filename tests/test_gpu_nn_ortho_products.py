"""The products of orthogonal updates against the same arithmetic in 64 bits: every kernel, in the last step and ahead of it, wide and tall."""
import pytest
import torch

import ortho_emulation as emulation
from ortho_sizes import SIZES

pytestmark = pytest.mark.gpu

TYPES = [(torch.float32, torch.float32), (torch.float16, torch.float16), (torch.float16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)]
IDS = ["f32", "f16", "f16-f32", "bf16", "bf16-f32"]
STEPS = 2
#: What SIZES does not reach both wide and tall.
MORE = [(16, 641, 545), (25, 706, 764)]


def both_parts(dtype, rows, cols):
    return dtype is not torch.bfloat16 or min(rows, cols) <= 256


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES + MORE, ids=lambda s: "x".join(map(str, s)))
def test_every_kernel(types, size):
    """Two usual steps, of gradients whose every term shows (test_ortho_emulation.py: a share of k or an eighth of a side that S S lacks is tens of tolerances off)."""
    from paper_2103_07454_amd import nn
    dtype, out_dtype = types
    W, R, C = size
    gen = torch.Generator(device="cuda").manual_seed(R + 3 * C)
    grad = emulation.gradient(gen, W, R, C).to(dtype)
    out = nn.Orthogonal(R, C, matrices=W, dtype=dtype, out_dtype=out_dtype, steps=STEPS, scale=-1.5).update(grad)
    for w in sorted({0, W // 2, W - 1}):
        u = grad[w].float()
        options = dict(steps=STEPS, scale=-1.5)
        want = emulation.emulate(u, both_parts(dtype, R, C), out_dtype, **options)
        room = emulation.tolerance(want, u, both_parts(dtype, R, C), out_dtype, **options)
        off, size_of = float((out[w].double() - want).norm()), float(want.norm())
        print(f"[ortho products] {size} {dtype} {out_dtype}: off by {off / size_of:.1e} of the update, {off / room:.2f} of the tolerance", flush=True)
        assert off <= room


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("size", [(2, 65, 130), (1, 333, 200), (1, 700, 512), (1, 899, 1089), (4, 128, 784)], ids=lambda s: "x".join(map(str, s)))
def test_the_usual_five_steps(types, size):
    from paper_2103_07454_amd import nn
    dtype, out_dtype = types
    W, R, C = size
    gen = torch.Generator(device="cuda").manual_seed(R + 5 * C)
    grad = emulation.gradient(gen, W, R, C).to(dtype)
    out = nn.Orthogonal(R, C, matrices=W, dtype=dtype, out_dtype=out_dtype).update(grad)
    for w in range(W):
        u = grad[w].float()
        want = emulation.emulate(u, both_parts(dtype, R, C), out_dtype)
        room = emulation.tolerance(want, u, both_parts(dtype, R, C), out_dtype)
        off, size_of = float((out[w].double() - want).norm()), float(want.norm())
        print(f"[ortho five] {size} {dtype} {out_dtype}: off by {off / size_of:.1e} of the update, {off / room:.2f} of the tolerance of {room / size_of:.1e}", flush=True)
        assert off <= room


@pytest.mark.parametrize("types", [TYPES[0], TYPES[3]], ids=[IDS[0], IDS[3]])
def test_matrices_beyond_32_bits(types):
    """The last matrix's X, gradient and update lie more than 2^32 bytes behind the first's."""
    from paper_2103_07454_amd import nn
    dtype, out_dtype = types
    W, R, C = (17 if dtype is torch.float32 else 33), 1024, 65536
    gen = torch.Generator(device="cuda").manual_seed(6)
    grad = torch.empty(W, R, C, dtype=dtype, device="cuda")
    for w in range(W):
        grad[w] = emulation.gradient(gen, 1, R, C)[0]
    momentum = torch.zeros(W, R, C, device="cuda")
    out = nn.Orthogonal(R, C, matrices=W, dtype=dtype, out_dtype=out_dtype, steps=STEPS, nesterov=False).update(grad, momentum=momentum)
    for w in (0, W - 1):
        u = grad[w].float()
        assert torch.equal(momentum[w], u)
        want = emulation.emulate(u, both_parts(dtype, R, C), out_dtype, steps=STEPS)
        assert float((out[w].double() - want).norm()) <= emulation.tolerance(want, u, both_parts(dtype, R, C), out_dtype, steps=STEPS)
