"""Layer norms of rows that lie far from 0: the unit row belongs to the spread of a row, not to where it lies."""
import pytest
import torch

import nn_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
SHORT = {torch.bfloat16: "bf16", torch.float16: "f16", torch.float32: "f32"}
EPS = 1e-5
# 1 / 117, 1 / 119 and 1 / 120 in 32 bits, times the width, are not 1; 16 to 1024 threads to a row, widths in eights and not
WIDTHS = [3, 117, 119, 120, 250, 488, 785, 1000, 2040, 4000, 4100, 8200]


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("width", WIDTHS)
def test_constant_rows(nn, dtype, width):
    """Rows whose sums, and all their partial sums, are exact: the unit row is 0 to the last bit."""
    op = nn.BlockNorm(width, max_rows=5, dtype=dtype, kind=nn.LAYER, eps=EPS)
    # few bits each: times a width of 13 bits they stay below 24
    value = torch.tensor([9984.0, -9984.0, 0.0, 1.25, 448.0], device="cuda").to(dtype)
    x = value[None, :, None].expand(1, 5, width).contiguous()
    w, b = torch.ones(1, width, dtype=dtype, device="cuda"), torch.full((1, width), 0.25, dtype=dtype, device="cuda")
    _, n = op.forward(x, pre=w, pre_bias=b)
    assert bool((n == 0.25).all())
    r, n = op.forward(torch.zeros_like(x), x, post=w, post_bias=b, pre=w)
    assert bool((r == 0.25).all()) and bool((n == 0).all())
    gen = torch.Generator(device="cuda").manual_seed(width)
    dn = torch.randn(1, 5, width, generator=gen, device="cuda").to(dtype)
    d = op.backward(None, dn, x, pre=w, pre_bias=b)
    assert bool((d["d_pre"] == 0).all())
    q = dn.double()
    want = (q - q.mean(-1, keepdim=True)) / EPS ** 0.5
    # the mean of q is held in 32 bits (26 roundings), the difference, the root and the product round once each
    bound = 32 * ref.U32 * (q.abs() + q.abs().mean(-1, keepdim=True)) / EPS ** 0.5
    assert bool(((d["d_residual"].double() - want).abs() <= bound + ref.rounding(want.abs() + bound, dtype)).all())
    d = op.backward(dn, None, torch.zeros_like(x), x, post=w, post_bias=b)
    assert bool((d["d_post"] == 0).all())


@pytest.mark.parametrize("width", WIDTHS[1:])
def test_rows_far_from_zero(nn, width):
    """Rows of 1e4 with a spread of 0.05, in 32 bits.

    x - mean is exact (the two are within a factor of 2), so what the mean is off by, at most 26 roundings of 1e4 or 0.3 of the
    spread, can be found from the differences' sum, which is off by 26 roundings of their size: at most 28 U32 (1 + |u|) of the unit row
    with the root and the quotient, and as much for the share of the variance that has to be taken back.  64 hold both."""
    rows = 6
    gen = torch.Generator().manual_seed(width)
    x = (1e4 + 0.05 * torch.randn(1, rows, width, generator=gen)).cuda()
    pre, bias = torch.randn(1, width, generator=gen).cuda(), torch.randn(1, width, generator=gen).cuda()
    dn = torch.randn(1, rows, width, generator=gen).cuda()
    op = nn.BlockNorm(width, max_rows=rows, dtype=torch.float32, kind=nn.LAYER, eps=EPS)
    u, inv = ref.unit("layer", x[0].double(), EPS)
    off_u = 64 * ref.U32 * (1 + u.abs())
    w, b, g = pre[0].double(), bias[0].double(), dn[0].double()

    def near(got, want, bound, what):
        off = (got.double() - want).abs()
        print(f"[norm] width {width} {what}: share of the bound {float((off / bound).max()):.2g}", flush=True)
        assert bool((off <= bound).all()), what

    _, n = op.forward(x, pre=pre, pre_bias=bias)
    near(n[0], u * w + b, off_u * w.abs() + 4 * ref.U32 * ((u * w).abs() + b.abs()), "normed")
    r, _ = op.forward(torch.zeros_like(x), x, post=pre, post_bias=bias)
    near(r[0], u * w + b, off_u * w.abs() + 4 * ref.U32 * ((u * w).abs() + b.abs()), "after")
    q = g * w
    size = q.abs() + q.abs().mean(-1, keepdim=True) + (1 + u.abs()) * (q * (1 + u.abs())).abs().mean(-1, keepdim=True)
    for d, name in ((op.backward(None, dn, x, pre=pre, pre_bias=bias), "residual"),
                    (op.backward(dn, None, torch.zeros_like(x), x, post=pre, post_bias=bias), "branch")):
        near(d["d_" + name][0], ref.unit_gradient("layer", q, u, inv), 128 * ref.U32 * inv * size, "d_" + name)
        near(d["d_pre" if name == "residual" else "d_post"][0], (g * u).sum(0), (g.abs() * (off_u + 8 * ref.U32 * u.abs())).sum(0), name + "'s weight")
