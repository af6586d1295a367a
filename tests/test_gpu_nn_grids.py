"""Calls of more workgroups than one grid takes (2^32 threads)."""
import math

import pytest
import torch

import nn_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    yield m
    torch.cuda.empty_cache()


def test_norms_of_many_rows(nn):
    """16 threads to a row, 2^28 rows and some: 4 GB each way."""
    T, D = 2 ** 28 + 4099, 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(1, T, D, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    w = torch.ones(1, D, dtype=torch.bfloat16, device="cuda")
    _, n = nn.BlockNorm(D, max_rows=T, eps=1e-5).forward(x, pre=w, normed=torch.full_like(x, 9.0))
    for a in range(0, T, 1 << 25):
        v = x[0, a:a + (1 << 25)].float()
        want = v / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-5)
        # two roundings to the type, and the 32-bit sums' own
        assert bool(((n[0, a:a + (1 << 25)].float() - want).abs() <= 1.01 * ref.UNIT[torch.bfloat16] * want.abs() + 1e-30).all()), a


def test_copies_of_many_rows(nn):
    """A width of 7 is copied row by row, a wavefront to a row: 2^26 rows and some."""
    T, D, F = 2 ** 26 + 1027, 7, 8
    gen = torch.Generator(device="cuda").manual_seed(2)
    make = lambda *s: torch.empty(*s, dtype=torch.float16, device="cuda").normal_(generator=gen).mul_(0.5)
    x, wg, wu, wd = make(1, T, D), make(1, F, D), make(1, F, D), make(1, D, F)
    y = nn.GatedFFN(D, F, max_rows=T, dtype=torch.float16).forward(x, wg, wu, wd)
    for a in (0, T // 2, T - 3000):
        part = slice(a, a + 3000)
        value, bound = ref.ffn("silu", torch.float16, x[0, part].double(), wg[0].double(), wu[0].double(), wd[0].double())["y"]
        assert bool(((y[0, part].double() - value).abs() <= bound).all()), a
    # the copies' last rows went with a second launch: all rows of one value give one result
    x[:] = 0.25
    y = nn.GatedFFN(D, F, max_rows=T, dtype=torch.float16).forward(x, wg, wu, wd)
    assert bool((y == y[:, :1]).all())


def test_products_of_many_workers(nn):
    """One token of each of 65535 workers, 1024 threads to eight columns of 520."""
    W, D, F = 65535, 520, 8
    gen = torch.Generator(device="cuda").manual_seed(3)
    make = lambda *s, size=1.0: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(generator=gen).mul_(size)
    t = dict(x=make(W, 1, D), w_gate=make(W, F, D, size=D ** -0.5), w_up=make(W, F, D, size=D ** -0.5), w_down=make(W, D, F, size=F ** -0.5))
    y = nn.GatedFFN(D, F, workers=W, max_rows=1).forward(*t.values())
    for w in [*range(40), W // 2, *range(W - 1100, W, 7), W - 1]:
        value, bound = ref.ffn("silu", torch.bfloat16, *(v[w].double() for v in t.values()))["y"]
        assert bool(((y[w].double() - value).abs() <= bound).all()), w


def test_clipping_many_short_tensors(nn):
    """20000 tensors of five elements for each of 1024 workers: as many sums."""
    P, L = 1024, 20_000
    op = nn.GradClip([5] * L, P)
    grad = torch.full((P, op.pitch), float("nan"), device="cuda")
    real = grad.view(P, -1)[:, :8 * L].view(P, L, 8)[:, :, :5]
    real.copy_(torch.randn(P, L, 5, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda"))
    out, norm = op.clip(grad, 1.0, out=torch.zeros_like(grad))
    want = real.double().square().sum((1, 2)).sqrt()
    assert bool(((norm.double() - want).abs() <= 2 * ref.U32 * want).all())
    clipped = real.double() / (want + 1e-6)[:, None, None]
    got = out[:, :8 * L].view(P, L, 8)
    assert bool(((got[:, :, :5].double() - clipped).abs() <= 8 * ref.U32 * clipped.abs()).all()) and float(got[:, :, 5:].abs().max()) == 0.0


def test_sums_of_many_workers(nn):
    """The weights' gradients of 1.1 million workers of one row: four sums of 64 columns each, 1024 threads to one."""
    W, D = 1_100_000, 16
    gen = torch.Generator(device="cuda").manual_seed(5)
    make = lambda *s: torch.empty(*s, device="cuda").normal_(generator=gen)
    x, pre, dn = make(W, 1, D), make(W, D), make(W, 1, D)
    d = nn.BlockNorm(D, workers=W, max_rows=1, dtype=torch.float32, eps=1e-5).backward(None, dn, x, pre=pre)
    u = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + 1e-5)
    # one row: the product and the unit row's few roundings
    assert bool(((d["d_pre"].double() - (dn * u)[:, 0]).abs() <= 16 * ref.U32 * (dn * u)[:, 0].abs() + 1e-30).all())
    assert math.isfinite(float(d["d_residual"].sum()))
