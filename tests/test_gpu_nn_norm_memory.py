"""What a norm's context takes of the GPU's memory: room for the backward pass's sums, as much as its stripes can need and only where there is one."""
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


def taken(make):
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    op = make()
    return op, before - torch.cuda.mem_get_info()[0]


@pytest.mark.parametrize("kind,slots", [("RMS", 3), ("LAYER", 5)])
def test_room_for_the_backward_pass(nn, kind, slots):
    """1024 stripes are aimed at, twice as many may come of the gate's groups, each with a row of sums for every weight and the gate."""
    op, memory = taken(lambda: nn.BlockNorm(4096, max_rows=1 << 20, kind=getattr(nn, kind)))
    assert memory <= 2 * 1024 * slots * 4096 * 4 + (4 << 20)
    op, memory = taken(lambda: nn.BlockNorm(16384, max_rows=3, kind=getattr(nn, kind)))
    assert memory <= 2 * 3 * slots * 16384 * 4 + (4 << 20)


def test_forward_only(nn):
    from paper_2103_07454_amd import evg
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(1, 40, 16384, generator=gen, device="cuda").bfloat16()
    w = torch.randn(1, 16384, generator=gen, device="cuda").bfloat16()
    op, memory = taken(lambda: nn.BlockNorm(16384, max_rows=1 << 16, train=False))
    assert memory <= 1 << 20
    got = op.forward(x, x, post=w, pre=w)
    want = nn.BlockNorm(16384, max_rows=40).forward(x, x, post=w, pre=w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(evg.EvgError) as e:
        op.backward(x, None, x, x, post=w, pre=w)
    assert e.value.status == 5


@pytest.mark.parametrize("workers,rows,gate_rows", [(1024, range(1, 26), range(1, 28)), (1, [2047, 2048, 2049, 4095, 4097, 6151, 9000],
                                                                                        [1, 2, 3, 4, 5, 6, 7, 1023, 1025, 2047, 2049, 4096, 5000])],
                         ids=["few stripes", "many stripes"])
def test_every_division_into_stripes_has_room(nn, workers, rows, gate_rows):
    """Four stripes a worker are aimed at, or 2048: all numbers of rows up to six times as many, and groups of all lengths around a stripe's.  The
    gate's gradient of 32-bit values without norms is a plain sum."""
    D = 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    for T in rows:
        b, d = (torch.randn(workers, T, D, generator=gen, device="cuda") for _ in range(2))
        for g in gate_rows:
            op = nn.BlockNorm(D, workers=workers, max_rows=T, dtype=torch.float32, gate_rows=g)
            n = -(-T // g)
            gate = torch.ones(workers, n, D, device="cuda")
            got = op.backward(d, None, torch.zeros_like(b), b, gate=gate)["d_gate"]
            terms = (b * d).double()
            padded = torch.zeros(workers, n * g, D, dtype=torch.float64, device="cuda")
            padded[:, :T] = terms
            want, size = padded.view(workers, n, g, D).sum(2), padded.abs().view(workers, n, g, D).sum(2)
            assert bool(((got.double() - want).abs() <= min(g, T) * 2.0 ** -24 * size + 1e-30).all()), (T, g)
