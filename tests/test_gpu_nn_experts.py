"""Tokens by expert and back against the definition in 64 bits, and the refusals."""
import pytest
import torch

import nn_experts_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
#: workers, tokens, experts, top, capacity, width: one token, one expert, all experts; room for none, some and all; odd widths and several column
#: blocks; more entries than one workgroup places; many experts
SIZES = [(1, 1, 1, 1, 0, 1), (1, 1, 8, 8, 0, 130), (1, 1, 8, 2, 3, 40), (3, 7, 5, 2, 0, 33), (3, 7, 5, 2, 2, 33), (2, 100, 4, 4, 0, 1030), (2, 100, 16, 3, 100, 24),
         (1, 65, 1000, 9, 1, 16), (1, 1000, 3, 1, 333, 8), (1, 5000, 7, 3, 0, 5), (2, 4097, 64, 3, 150, 9), (1, 20_001, 1024, 1, 0, 3), (2, 0, 3, 2, 4, 8), (2, 0, 3, 2, 0, 8)]


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


def within(got, want, what):
    value, bound = want
    off = (got.double().cpu() - value).abs()
    assert bool((off <= bound).all()), f"{what}: {float((off - bound).max())} beyond the bound"


def choices(gen, W, T, E, K, none=0.2):
    """Different experts for each token, in any order; some places have none, some numbers that there are not."""
    chosen = torch.rand(W, T, E, generator=gen).argsort(-1)[..., :K].int()
    miss = torch.rand(W, T, K, generator=gen)
    chosen[miss < none] = -1
    chosen[miss > 0.98] = E
    chosen[miss > 0.99] = -2 ** 31
    return chosen


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_definition(nn, dtype, size):
    W, T, E, K, C, D = size
    gen = torch.Generator().manual_seed(T + E + C)
    op = nn.ExpertSort(E, K, D, workers=W, max_tokens=T + 2, capacity=C, dtype=dtype)
    S = op.slots(T)
    make = lambda *s: torch.randn(*s, generator=gen).to(dtype)  # noqa: E731
    chosen, x, done, dy, d_in = choices(gen, W, T, E, K), make(W, T, D), make(W, S, D), make(W, T, D), make(W, S, D)
    weights = torch.randn(W, T, K, generator=gen)
    rows, plan = op.dispatch(x.cuda(), chosen.cuda(), rows=torch.full((W, S, D), float("nan"), dtype=dtype, device="cuda"))
    y = op.combine(done.cuda(), weights.cuda(), plan)
    dx = op.dispatch_backward(d_in.cuda(), plan)
    d_done, d_weights = op.combine_backward(dy.cuda(), done.cuda(), weights.cuda(), plan,
                                            d_rows=torch.full((W, S, D), float("nan"), dtype=dtype, device="cuda"))
    alone = op.combine_backward(dy.cuda(), done.cuda(), weights.cuda(), plan, weight_gradients=False)
    assert alone[1] is None and torch.equal(alone[0], d_done)
    alone = op.combine_backward(dy.cuda(), done.cuda(), weights.cuda(), plan, row_gradients=False)
    assert alone[0] is None and torch.equal(alone[1], d_weights)
    for w in range(W):
        slot, source, counts = ref.plan(chosen[w], E, C)
        assert torch.equal(plan.slot[w].cpu(), slot) and torch.equal(plan.source[w].cpu(), source) and torch.equal(plan.counts[w].cpu(), counts)
        assert torch.equal(rows[w].cpu(), ref.dispatch(x[w], source, K))
        within(y[w], ref.combine(done[w].double(), weights[w].double(), slot, dtype), "y")
        within(dx[w], ref.combine(d_in[w].double(), None, slot, dtype), "dx")
        a, b = ref.combine_backward(dy[w].double(), done[w].double(), weights[w].double(), slot, source, K, dtype)
        within(d_done[w], a, "d_rows")
        within(d_weights[w], b, "d_weights")


@pytest.mark.parametrize("entries", [8192, 8193], ids=["one-workgroup", "many"])
def test_order_is_kept_where_all_go_to_one_expert(nn, entries):
    op = nn.ExpertSort(5, 1, 1, max_tokens=entries, dtype=torch.float32)
    x = torch.arange(entries, dtype=torch.float32, device="cuda").view(1, entries, 1)
    rows, plan = op.dispatch(x, torch.full((1, entries, 1), 3, dtype=torch.int32, device="cuda"))
    assert torch.equal(rows, x) and plan.counts[0].tolist() == [0, 0, 0, entries, 0]
    # the same expert twice: two entries
    two = nn.ExpertSort(2, 2, 1, max_tokens=4, dtype=torch.float32)
    rows, plan = two.dispatch(x[:, :4], torch.ones(1, 4, 2, dtype=torch.int32, device="cuda"))
    assert rows[0, :, 0].tolist() == [0, 0, 1, 1, 2, 2, 3, 3] and two.dispatch_backward(rows, plan)[0, :, 0].tolist() == [0, 2, 4, 6]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_strides_and_what_lies_beside(nn, dtype):
    W, T, E, K, C, D = 2, 50, 4, 2, 20, 19
    gen = torch.Generator().manual_seed(4)
    op = nn.ExpertSort(E, K, D, workers=W, max_tokens=T, capacity=C, dtype=dtype)
    chosen = choices(gen, W, T, E, K).cuda()
    x = torch.randn(T, W, D + 3, generator=gen).to(dtype).cuda().transpose(0, 1)[..., 1:1 + D]
    weights = torch.randn(W, T, K, generator=gen).cuda()
    want, plan = op.dispatch(x.contiguous(), chosen)
    room = torch.full((W, E * C + 1, D + 2), 7.0, dtype=dtype, device="cuda")
    rows, _ = op.dispatch(x, chosen, rows=room[:, 1:, 1:1 + D], plan=plan)
    assert torch.equal(rows, want)
    room[:, 1:, 1:1 + D] = 7.0
    assert bool((room == 7.0).all())
    out = torch.full((W, T, D + 1), 7.0, dtype=dtype, device="cuda")
    y = op.combine(want, weights, plan)
    assert torch.equal(op.combine(want, weights, plan, out=out[..., 1:]), y) and bool((out[..., 0] == 7).all())
    d, dw = op.combine_backward(x, want, weights, plan, d_rows=room[:, 1:, 1:1 + D])
    d2, dw2 = op.combine_backward(x.contiguous(), want.clone(), weights, plan)
    assert torch.equal(d, d2) and torch.equal(dw, dw2)
    one = x[:, :1].expand(W, T, D)          # one row for all tokens
    assert torch.equal(op.dispatch(one, chosen)[0], op.dispatch(one.contiguous(), chosen)[0])


def test_values_that_are_not_finite_stay_where_they_are(nn):
    """What lies in empty slots and at places that are left out is not read."""
    op = nn.ExpertSort(3, 2, 4, max_tokens=5, capacity=2, dtype=torch.float32)
    chosen = torch.tensor([[[0, 1], [0, -1], [0, 2], [-1, -1], [1, 2]]], dtype=torch.int32, device="cuda")
    x = torch.ones(1, 5, 4, device="cuda")
    x[0, 3] = float("nan")                      # goes nowhere
    rows, plan = op.dispatch(x, chosen)
    assert torch.isfinite(rows).all() and plan.counts[0].tolist() == [3, 2, 2]
    done = torch.full_like(rows, float("nan"))
    done[0, plan.source[0] >= 0] = 1.0
    weights = torch.where(plan.slot >= 0, 1.0, float("nan"))
    y = op.combine(done, weights, plan)
    assert y[0, :, 0].tolist() == [2, 1, 1, 0, 2]
    d, dw = op.combine_backward(torch.ones_like(x), done, weights, plan)
    assert torch.isfinite(d).all() and dw[0].tolist() == [[4, 4], [4, 0], [0, 4], [0, 0], [4, 4]]


def test_rows_beyond_32_bits(nn):
    T, D = 300_000, 8192
    op = nn.ExpertSort(2, 1, D, max_tokens=T, dtype=torch.bfloat16)
    x = torch.zeros(1, T, D, dtype=torch.bfloat16, device="cuda")
    x[0, 0, 5], x[0, T - 1, D - 1] = 3.0, 2.0
    chosen = torch.ones(1, T, 1, dtype=torch.int32, device="cuda")
    chosen[0, T - 1] = 0
    rows, plan = op.dispatch(x, chosen)
    assert float(rows[0, 0, D - 1]) == 2.0 and float(rows[0, 1, 5]) == 3.0 and int(plan.slot[0, 0, 0]) == 1
    y = op.dispatch_backward(rows, plan, dx=x)
    assert float(y[0, 0, 5]) == 3.0 and float(y[0, T - 1, D - 1]) == 2.0 and int((y != 0).sum()) == 2


def test_refusals(nn):
    from paper_2103_07454_amd import evg
    op = nn.ExpertSort(3, 2, 4, workers=2, max_tokens=5, capacity=4, dtype=torch.float32)
    x, chosen, w = torch.zeros(2, 5, 4, device="cuda"), torch.zeros(2, 5, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, 5, 2, device="cuda")
    rows, plan = op.dispatch(x, chosen)
    for bad in (x[:1], x.half(), torch.zeros(2, 6, 4, device="cuda"), x[..., :3]):
        with pytest.raises(ValueError):
            op.dispatch(bad, chosen)
    for bad in (chosen.long(), chosen[:, :4], chosen.cpu()):
        with pytest.raises(ValueError):
            op.dispatch(x, bad)
    with pytest.raises(ValueError):
        op.combine(rows[:, :11], w, plan)
    with pytest.raises(ValueError):
        op.combine(rows, w[:, :4], plan)
    with pytest.raises(ValueError):
        op.combine(rows, w, plan._replace(slot=plan.slot[:, :4]))
    with pytest.raises(ValueError):
        op.combine(rows, w, nn.ExpertPlan(plan.slot.view(-1), plan.source, plan.counts))
    for call in (lambda: op.dispatch(rows[:, :5], chosen, rows=rows), lambda: op.combine(rows, w, plan, out=rows[:, :5]),
                 lambda: op.combine_backward(x, rows, w, plan, d_rows=rows), lambda: op.combine_backward(x, rows, w, plan, d_weights=w),
                 lambda: nn.ExpertSort(2, 3, 4, max_tokens=5), lambda: nn.ExpertSort(1025, 3, 4, max_tokens=5), lambda: nn.ExpertSort(1000, 3, 4, max_tokens=5, capacity=1 << 22),
                 lambda: nn.ExpertSort(4, 3, 0, max_tokens=5), lambda: nn.ExpertSort(4, 4, 4, max_tokens=1 << 26)):
        with pytest.raises(evg.EvgError):
            call()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("width", [2048, 1100])
def test_rows_that_the_caches_do_not_hold(nn, dtype, width):
    """More than 128 MB of rows, with room for some: every kernel that moves them past the caches."""
    T, E, K = 40_003, 6, 2
    gen = torch.Generator(device="cuda").manual_seed(5)
    op = nn.ExpertSort(E, K, width, max_tokens=T, capacity=12_000, dtype=dtype)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    x, dy, done = make(1, T, width), make(1, T, width), make(1, E * 12_000, width)
    weights = torch.randn(1, T, K, generator=gen, device="cuda")
    chosen = torch.rand(1, T, E, generator=gen, device="cuda").argsort(-1)[..., :K].int()
    rows, plan = op.dispatch(x, chosen)
    slot, source, counts = ref.plan(chosen[0].cpu(), E, 12_000)
    assert torch.equal(plan.slot[0].cpu(), slot) and torch.equal(plan.source[0].cpu(), source) and int(counts.max()) > 12_000 > int(counts.min()) - 2_000
    y, (d_done, d_weights) = op.combine(done, weights, plan), op.combine_backward(dy, done, weights, plan)
    some = torch.cat([torch.arange(50), torch.randint(0, T, (400,)), torch.arange(T - 50, T)])
    at = slot[some]
    within(y[0, some.cuda()], ref.combine(done[0].cpu().double(), weights[0, some.cuda()].cpu().double(), at, dtype), "y")
    real = (source >= 0).cuda()
    token = source.cuda().long().clamp(min=0) // K
    assert torch.equal(rows[0], torch.where(real[:, None], x[0, token], torch.zeros((), dtype=dtype, device="cuda")))
    w = weights.view(-1)[source.cuda().long().clamp(min=0)]
    # The product of 24 and at most 24 bits is exact in 64.  It is rounded to 32 bits and then to the type, or to the type at once (float16 products have an
    # instruction for that): U32 and a rounding of the type cover both, where bits need not be the same, as a value that the first rounding takes to the middle
    # between two neighbours may go either way in the second.
    want = torch.where(real[:, None], w[:, None].double() * dy[0, token].double(), 0.0)
    off = (d_done[0].double() - want).abs()
    assert bool((off <= ref.U32 * want.abs() + ref.rounding(want, dtype)).all())
    del want, off
    terms = torch.where((at >= 0)[..., None], dy[0].cpu().double()[some][:, None] * done[0].cpu().double()[at.long().clamp(min=0)], 0.0)
    within(d_weights[0, some.cuda()], (terms.sum(-1), (width + 1) * ref.U32 * terms.abs().sum(-1)), "d_weights")
