"""Orthogonal updates against the formula in 64 bits, and their refusals."""
import math

import pytest
import torch

import nn_experts_reference as ref
import nn_reference
from ortho_sizes import SIZES as EVERY_TILE

pytestmark = pytest.mark.gpu

TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float16, torch.float32)]
IDS = ["f32", "bf16", "bf16-f32", "f16", "f16-f32"]
#: A matrix with the sides' order, odd and whole sizes, one row, one column; every tile, and several of each
SIZES = [(1, 1, 1), (1, 1, 7), (1, 9, 1), (2, 3, 5), (3, 17, 8), (2, 64, 64), (2, 65, 130), (1, 130, 65), (2, 200, 333), (1, 333, 200), (1, 40, 1000), (1, 1000, 40)]
#: A step that hardly stretches anything, so that bounds stay tight over several: singular values s to 1.5 s - 0.5 s^3, and to the quintic
#: that is flat at 1
GENTLE = [(1.5, -0.5, 0.0), (1.875, -1.25, 0.375)]


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


def gradient(gen, *shape):
    """A few directions carry most of it."""
    w, r, c = shape
    k = max(1, min(r, c) // 8)
    return 1e-3 * (torch.bmm(torch.randn(w, r, k, generator=gen), torch.randn(w, k, c, generator=gen)) / k ** 0.5 + 0.3 * torch.randn(w, r, c, generator=gen))


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("steps,polynomial", [(1, ref.POLYNOMIAL), (2, GENTLE[0]), (3, GENTLE[1]), (4, GENTLE[0])])
def test_against_the_formula(nn, types, size, steps, polynomial):
    dtype, out_dtype = types
    W, R, C = size
    gen = torch.Generator().manual_seed(R * C + steps)
    grad, old = gradient(gen, W, R, C).to(dtype), 5 * gradient(gen, W, R, C)
    op = nn.Orthogonal(R, C, matrices=W, dtype=dtype, out_dtype=out_dtype, steps=steps, polynomial=polynomial, momentum=0.9, nesterov=steps != 2, scale=-2.0)
    new = torch.full((W, R, C), 7.0, device="cuda")
    out = op.update(grad.cuda(), momentum=old.cuda(), momentum_out=new)
    plain = op.update(grad.cuda())
    assert out.dtype == out_dtype and out.shape == (W, R, C)
    for w in range(W):
        m, u = ref.momentum(grad[w].double(), old[w].double(), float(torch.tensor(0.9)), steps != 2)
        # one product and one sum in 32 bits, at most two roundings
        assert bool(((new[w].double().cpu() - m).abs() <= 2 * ref.U32 * (0.9 * old[w].double().abs() + grad[w].double().abs()) + 2.0 ** -149).all())
        for got, of in ((out[w], u), (plain[w], grad[w].double())):
            want, bound = ref.orthogonal(of, dtype, steps=steps, polynomial=polynomial, scale=-2.0)
            bound += float(nn_reference.rounding(want.abs() + 1e-3, out_dtype).norm())
            off = float((got.double().cpu() - want).norm())
            assert off <= bound, (off, bound, float(want.norm()))


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("size", [(1, 512, 700), (1, 700, 512), (2, 1100, 1024), (9, 300, 300)], ids=lambda s: "x".join(map(str, s)))
def test_larger_tiles(nn, types, size):
    dtype, out_dtype = types
    W, R, C = size
    gen = torch.Generator().manual_seed(7)
    grad = gradient(gen, W, R, C).to(dtype)
    out = nn.Orthogonal(R, C, matrices=W, dtype=dtype, out_dtype=out_dtype, steps=2, polynomial=GENTLE[0]).update(grad.cuda())
    for w in range(0, W, 4):
        want, bound = ref.orthogonal(grad[w].double(), dtype, steps=2, polynomial=GENTLE[0])
        bound += float(nn_reference.rounding(want.abs() + 1e-3, out_dtype).norm())
        assert float((out[w].double().cpu() - want).norm()) <= bound


def one_step(u, dtype, polynomial):
    """A step's result and a bound of each element.  With X of norm 1, r its rows' norms and c its columns' (wide; tall the other way round), p those of P's rows,
    o an operand's rounding, and sums of absolute products at most the products of norms:
        |dS_ij| <= E r_i r_j,  E = 3 o + k 2^-24                                       (two operands, the result, the sum)
        |dP_ij| <= Q r_i r_j + o |P_ij|,  Q = |b| E + |c| (2 E + 2 o + n 2^-24)
        |dX'_ij| <= |a| (2^-22 + 2^-24) |X_ij| + c_j (Q r_i + (2 o + n 2^-24) p_i)
    and what the start is off, d = 4 * 2^-24 + 2^-22 of each element, comes to d (|a X_ij| + (3 |b| + 5 |c|) r_i c_j) at most.
    """
    a, b, c = polynomial
    o, d = 2 * ref.KEPT if dtype == torch.float32 else ref.HALF, 4 * ref.U32 + ref.KEPT
    x = u / (u.norm() + 1e-7)
    if x.shape[0] > x.shape[1]:
        out, bound = one_step(u.T, dtype, polynomial)
        return out.T, bound.T
    n, k = x.shape
    S = x @ x.T
    P = b * S + c * S @ S
    E = 3 * o + k * ref.U32
    Q = abs(b) * E + abs(c) * (2 * E + 2 * o + n * ref.U32)
    r, cols, p = x.norm(dim=1)[:, None], x.norm(dim=0)[None], P.norm(dim=1)[:, None]
    bound = abs(a) * (ref.KEPT + ref.U32) * x.abs() + cols * (Q * r + (2 * o + n * ref.U32) * p) + d * (abs(a) * x.abs() + (3 * abs(b) + 5 * abs(c)) * r * cols)
    return a * x + P @ x, 1.05 * bound


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", EVERY_TILE, ids=lambda s: "x".join(map(str, s)))
def test_every_tile(nn, dtype, size):
    """Products of hi alone (bfloat16) and of both parts (float32), of every tile, whole and in parts of k."""
    W, R, C = size
    gen = torch.Generator(device="cuda").manual_seed(R)
    k = max(1, min(R, C) // 8)
    grad = (torch.bmm(torch.randn(W, R, k, generator=gen, device="cuda"), torch.randn(W, k, C, generator=gen, device="cuda")) / k ** 0.5
            + 0.3 * torch.randn(W, R, C, generator=gen, device="cuda")).to(dtype)
    out = nn.Orthogonal(R, C, matrices=W, dtype=dtype, out_dtype=torch.float32, steps=1).update(grad)
    for w in range(W):
        want, bound = one_step(grad[w].double(), dtype, ref.POLYNOMIAL)
        off = (out[w].double() - want).abs()
        print(f"[ortho] {size} {dtype}: off by {float((off / bound).max()):.3f} of the bound, which is {float((bound / want.abs()).median()):.1e} of an element", flush=True)
        assert bool((off <= bound + nn_reference.rounding(want, torch.float32)).all())


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("size", [(96, 160), (160, 96), (128, 128)], ids=lambda s: "x".join(map(str, s)))
def test_five_steps_make_singular_values_alike(nn, types, size):
    dtype, out_dtype = types
    R, C = size
    gen = torch.Generator().manual_seed(8)
    grad = gradient(gen, 1, R, C).to(dtype)
    out = nn.Orthogonal(R, C, dtype=dtype, out_dtype=out_dtype).update(grad.cuda())
    want, bound = ref.orthogonal(grad[0].double(), dtype)
    off = float((out[0].double().cpu() - want).norm())
    assert off <= bound + float(nn_reference.rounding(want.abs() + 1e-3, out_dtype).norm())
    got = torch.linalg.svdvals(out[0].double().cpu())
    # p takes 0.27 .. 1.21 into 0.67 .. 1.21, and the larger singular values of a normed matrix have got there in five steps
    assert float(got.max()) < 1.25 and float(got[:R // 2].min()) > 0.65


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_places(nn, types):
    """In place, strides, odd addresses, one gradient for all matrices; what lies beside stays."""
    dtype, out_dtype = types
    W, R, C = 3, 20, 45
    gen = torch.Generator().manual_seed(9)
    op = nn.Orthogonal(R, C, matrices=W, dtype=dtype, out_dtype=out_dtype, steps=3, momentum=0.5)
    room = torch.full((R, W, C + 4), 7.0, dtype=dtype, device="cuda")
    grad = room.transpose(0, 1)[..., 3:3 + C]
    grad.copy_(gradient(gen, W, R, C))
    old = gradient(gen, W, R, C).cuda()
    want_m = torch.empty_like(old)
    want = op.update(grad.contiguous(), momentum=old, momentum_out=want_m)
    out = torch.full((W, R, C + 1), 7.0, dtype=out_dtype, device="cuda")
    mine = old.clone()
    got = op.update(grad, momentum=mine, out=out[..., 1:])
    assert torch.equal(got, want) and torch.equal(mine, want_m) and bool((out[..., 0] == 7).all())
    if dtype == out_dtype:
        assert torch.equal(op.update(grad, momentum=old.clone(), out=grad), want)
        assert bool((room[..., :3] == 7).all()) and bool((room[..., 3 + C:] == 7).all())
    shared = op.update(want[:1].to(dtype).expand(W, R, C))
    assert torch.equal(shared[0], shared[2])


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_zeros_and_what_is_not_finite(nn, types):
    dtype, out_dtype = types
    grad = torch.randn(4, 30, 70, device="cuda").to(dtype)
    grad[0] = 0
    grad[1, 3, 5] = float("nan")
    grad[3, 3, 5] = float("inf")
    for eps in (0.0, 1e-7):
        out = nn.Orthogonal(30, 70, matrices=4, dtype=dtype, out_dtype=out_dtype, eps=eps).update(grad)
        assert float(out[0].abs().max()) == 0.0 and torch.isnan(out[1]).all() and torch.isfinite(out[2]).all() and torch.isnan(out[3]).all()


@pytest.mark.parametrize("size", [1e-30, 1e25])
def test_sizes_of_gradients_do_not_matter(nn, size):
    """The sum of squares is held in 64 bits: neither 1e-60 nor 1e50 is lost."""
    grad = torch.randn(1, 40, 60, device="cuda")
    op = nn.Orthogonal(40, 60, eps=0.0)
    a, b = op.update(grad), op.update(grad * size)
    # the elements are rounded once more by the scaling, which five steps stretch like any other 2^-24 of each
    want, bound = ref.orthogonal(grad[0].double().cpu(), torch.float32, eps=0.0)
    assert float((a - b).double().norm()) <= 2 * bound


def test_refusals(nn):
    from paper_2103_07454_amd import evg
    op = nn.Orthogonal(4, 6, matrices=2)
    g, m = torch.zeros(2, 4, 6, device="cuda"), torch.zeros(2, 4, 6, device="cuda")
    for call in (lambda: op.update(g[:1]), lambda: op.update(g.half()), lambda: op.update(g, momentum=m.half()), lambda: op.update(g, momentum_out=m),
                 lambda: op.update(g, out=m.half()), lambda: op.update(g.transpose(1, 2)), lambda: nn.Orthogonal(4, 6, dtype=torch.float16, out_dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: op.update(g, momentum=g, momentum_out=m, out=m), lambda: op.update(g, momentum=m, momentum_out=g), lambda: op.update(g, momentum=m, out=m),
                 lambda: op.update(g, out=m[:1].expand(2, 4, 6)), lambda: nn.Orthogonal(4, 6, steps=0), lambda: nn.Orthogonal(4, 6, steps=65),
                 lambda: nn.Orthogonal(4, 6, polynomial=(4.0, 1.0, 1.0)), lambda: nn.Orthogonal(4, 6, polynomial=(float("nan"), 1.0, 1.0)),
                 lambda: nn.Orthogonal(20000, 17000), lambda: nn.Orthogonal(4, 6, eps=-1.0), lambda: nn.Orthogonal(4, 6, momentum=math.inf)):
        with pytest.raises(evg.EvgError):
            call()
