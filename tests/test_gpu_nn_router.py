"""Which experts tokens go to, their weights and the logits' gradient, against the definition in 64 bits, and the refusals."""
import math

import pytest
import torch

import nn_experts_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
#: experts, top: every number of lanes, first and last expert of each, all chosen, one chosen
SIZES = [(1, 1), (2, 1), (8, 8), (9, 2), (16, 3), (17, 4), (32, 5), (60, 4), (64, 8), (65, 8), (128, 8), (129, 6), (256, 8), (300, 9), (512, 4), (513, 2), (1000, 12), (1024, 1024)]


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


def within(got, want, what):
    value, bound = want
    off = (got.double().cpu() - value).abs()
    assert bool((off <= bound).all()), f"{what}: {float((off - bound).max())} beyond the bound"


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "of".join(map(str, reversed(s))))
@pytest.mark.parametrize("over_chosen", [False, True], ids=["all", "chosen"])
def test_against_the_definition(nn, dtype, size, over_chosen):
    E, K = size
    W, T = 2, 37
    gen = torch.Generator().manual_seed(E + K)
    logits = (2 * torch.randn(W, T, E, generator=gen)).to(dtype)
    logits[:, 5:15][torch.rand(W, 10, E, generator=gen) < 0.5] = -math.inf
    logits[:, 15] = -math.inf                                 # a row that nothing is left of
    logits[:, 16] = 1.0                                       # nothing but ties
    logits[:, 17] = torch.where(torch.rand(W, E, generator=gen) < 0.5, 0.0, -0.0).to(dtype)      # the two zeros are one value
    logits[:, 18] *= 20                                       # weights that vanish
    logits[:, 19] = torch.finfo(dtype).min                    # a mask of the type's lowest value is no mask: these are chosen
    logits[:, 20, : E // 2] = torch.finfo(dtype).min
    dw = torch.randn(W, T, K, generator=gen)
    op = nn.Router(E, K, workers=W, max_tokens=T + 5, dtype=dtype, over_chosen=over_chosen)
    chosen, weights = op.forward(logits.cuda())
    want = ref.choose(logits.double(), K)
    assert torch.equal(chosen.cpu(), want)
    d = op.backward(dw.cuda(), logits.cuda(), chosen)
    w, ew, g, eg = ref.route(logits.double(), want, over_chosen, dw.double(), dtype)
    within(weights, (w, ew), "weights")
    within(d, (g, eg), "d_logits")
    assert bool((d.cpu()[:, 15] == 0).all()) and bool((weights.cpu()[want < 0] == 0).all())


def test_what_is_not_finite(nn):
    """A NaN is chosen first and shows in the weights of its row alone; plus infinity as well."""
    logits = torch.zeros(1, 4, 6, device="cuda")
    logits[0, 1, 3] = float("nan")
    logits[0, 1, 5] = -float("nan")
    logits[0, 2, 4] = float("inf")
    for over_chosen in (False, True):
        op = nn.Router(6, 2, max_tokens=4, over_chosen=over_chosen)
        chosen, weights = op.forward(logits)
        assert chosen[0].tolist() == [[0, 1], [3, 5], [4, 0], [0, 1]]
        assert torch.isfinite(weights[0, [0, 3]]).all() and torch.isnan(weights[0, 1]).all() and torch.isnan(weights[0, 2, 0])
        d = op.backward(torch.ones_like(weights), logits, chosen)
        assert torch.isfinite(d[0, [0, 3]]).all() and torch.isnan(d[0, 1, 3])


def test_what_lies_at_unchosen_places_does_not_count(nn):
    logits = torch.full((1, 2, 5), -math.inf, device="cuda")
    logits[0, 0, 2] = 1.0
    op = nn.Router(5, 3, max_tokens=2)
    chosen, weights = op.forward(logits)
    assert chosen[0].tolist() == [[2, -1, -1], [-1, -1, -1]] and weights[0].tolist() == [[1, 0, 0], [0, 0, 0]]
    dw = torch.full((1, 2, 3), float("nan"), device="cuda")
    dw[0, 0, 0] = 3.0
    assert float(op.backward(dw, logits, chosen).abs().max()) == 0.0


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_strides_places_and_broadcasts(nn, dtype):
    gen = torch.Generator().manual_seed(1)
    W, T, E, K = 3, 9, 21, 4
    room = torch.randn(T, W, E + 4, generator=gen).to(dtype).cuda()
    logits = room.transpose(0, 1)[..., 3:3 + E]
    op = nn.Router(E, K, workers=W, max_tokens=T, dtype=dtype)
    plain = logits.contiguous()
    chosen, weights = op.forward(logits)
    again = op.forward(plain)
    assert torch.equal(chosen, again[0]) and torch.equal(weights, again[1])
    dw = torch.randn(W, T, K, generator=gen).cuda()
    want = op.backward(dw, plain, chosen)
    out = torch.full((W, T, E + 1), 7.0, dtype=dtype, device="cuda")
    assert torch.equal(op.backward(dw, logits, chosen, out=out[..., 1:]), want) and bool((out[..., 0] == 7).all())
    mine = plain.clone()
    assert op.backward(dw, mine, chosen, out=mine) is mine and torch.equal(mine, want)        # in place
    one = plain[:1, :1].expand(W, T, E)
    assert bool((op.forward(one)[0] == chosen[0, 0]).all())
    none = op.forward(plain[:, :0])
    assert none[0].shape == (W, 0, K) and op.backward(dw[:, :0].contiguous(), plain[:, :0], none[0]).shape == (W, 0, E)


def test_many_tokens(nn):
    """More workgroups than the chip holds, the last one in part."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.randn(1, 100_003, 8, generator=gen, device="cuda")
    chosen, weights = nn.Router(8, 2, max_tokens=100_003).forward(logits)
    best, at = logits.topk(2, dim=-1)
    assert torch.equal(chosen.long(), at) and torch.allclose(weights, torch.softmax(best, -1), rtol=1e-5)


def test_refusals(nn):
    from paper_2103_07454_amd import evg
    op = nn.Router(6, 2, workers=2, max_tokens=4)
    logits, chosen, w = torch.zeros(2, 4, 6, device="cuda"), torch.zeros(2, 4, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, 4, 2, device="cuda")
    for bad in (logits[:1], logits.half(), logits[..., :5], logits.cpu(), torch.zeros(2, 5, 6, device="cuda")):
        with pytest.raises(ValueError):
            op.forward(bad)
    for bad in (dict(chosen=chosen.long()), dict(chosen=chosen[:, :3]), dict(weights=w.half()), dict(weights=w.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            op.forward(logits, **bad)
    with pytest.raises(ValueError):
        op.backward(w[..., :1], logits, chosen)
    for call in (lambda: op.forward(logits, weights=logits.view(-1)[:16].view(2, 4, 2)), lambda: nn.Router(1025, 2, max_tokens=4), lambda: nn.Router(4, 5, max_tokens=4),
                 lambda: nn.Router(4, 0, max_tokens=4)):
        with pytest.raises(evg.EvgError):
            call()
