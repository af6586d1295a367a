"""The gated feed-forward block against its definition in 64 bits (bounds: tests/nn_reference.py), and its refusals."""
import pytest
import torch

import nn_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
SHORT = {torch.bfloat16: "bf16", torch.float16: "f16", torch.float32: "f32"}


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


def tensors(W, T, D, F, dtype, seed=0, device="cuda"):
    gen = torch.Generator().manual_seed(seed)
    make = lambda *s, size=1.0: (torch.randn(*s, generator=gen) * size).to(dtype).to(device)
    return dict(x=make(W, T, D), w_gate=make(W, F, D, size=D ** -0.5), w_up=make(W, F, D, size=D ** -0.5),
                w_down=make(W, D, F, size=F ** -0.5), dy=make(W, T, D))


def check(kind, dtype, t, got, names, device="cpu"):
    worst = {}
    for w in range(t["x"].shape[0]):
        v = {k: t[k][w].detach().to(device).double() for k in t}
        want = ref.ffn(kind, dtype, v["x"], v["w_gate"], v["w_up"], v["w_down"], v["dy"])
        for name in names:
            value, bound = want[name]
            off = (got[name][w].to(device).double() - value).abs()
            assert torch.isfinite(got[name][w]).all(), name
            worst[name] = max(worst.get(name, 0.0), float((off / bound).max()) if off.numel() else 0.0)
    print(f"\n[ffn] {SHORT[dtype]} {kind} {tuple(t['x'].shape)} hidden {t['w_gate'].shape[1]}: share of the bound "
          + ", ".join(f"{k} {v:.2g}" for k, v in worst.items()), flush=True)
    assert all(v <= 1.0 for v in worst.values()), worst


def train(nn, t, dtype, kind, **kw):
    W, T, D = t["x"].shape
    op = nn.GatedFFN(D, t["w_gate"].shape[1], workers=W, max_rows=T, dtype=dtype, activation=nn.ACTIVATIONS[kind], train=True)
    y, saved = op.forward(t["x"], t["w_gate"], t["w_up"], t["w_down"], save=True)
    dx, dg, du, dd = op.backward(t["dy"], t["x"], t["w_gate"], t["w_up"], t["w_down"], saved, **kw)
    return op, dict(y=y, dx=dx, dw_gate=dg, dw_up=du, dw_down=dd)


NAMES = ("y", "dx", "dw_gate", "dw_up", "dw_down")
# one token, lengths around the tiles' 64, 128 and 256, widths and hidden widths around a unit's 8, a step's 64 and a tile's edge
SIZES = [(1, 1, 64, 64), (1, 1, 1, 1), (1, 2, 8, 8), (2, 3, 7, 5), (1, 63, 64, 65), (1, 64, 72, 128), (1, 65, 120, 136), (3, 129, 96, 63),
         (1, 257, 200, 257), (2, 16, 264, 520), (1, 17, 130, 66), (1, 40, 512, 72), (5, 33, 40, 24),
         # long sums over few tiles, odd widths of more tokens than go straight from the tensors, padding of more than a small tile
         (1, 8, 1000, 520), (3, 9, 263, 1000), (1, 4, 2500, 3001), (1, 70, 1000, 96), (2, 70, 65, 33), (1, 300, 130, 263), (1, 90, 520, 1032), (2, 100, 7, 1030), (4, 100, 784, 203)]


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_backward(nn, dtype, size):
    t = tensors(*size, dtype)
    _, got = train(nn, t, dtype, "silu")
    check("silu", dtype, t, got, NAMES)


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "relu"])
def test_activations(nn, dtype, kind):
    t = tensors(2, 50, 136, 200, dtype, seed=1)
    _, got = train(nn, t, dtype, kind)
    # where ReLU's argument is not certain to be on one side, the slope may be either; the bound says so
    check(kind, dtype, t, got, NAMES)


@pytest.mark.parametrize("dtype,size", [(d, (1, 2100, 2056, 2312)) for d in TYPES] + [(d, s) for d in TYPES[:2] for s in ((1, 2600, 2560, 2600), (1, 3208, 3200, 3210))],
                         ids=lambda v: SHORT.get(v, str(v)) if isinstance(v, torch.dtype) else str(v))
def test_large_tiles(nn, dtype, size):
    """Sizes at which the larger tiles are chosen, for every product, with edges inside them."""
    t = tensors(*size, dtype, seed=2)
    _, got = train(nn, t, dtype, "silu")
    check("silu", dtype, t, got, NAMES, device="cuda")


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("size", [(1, 2000, 392, 648), (1, 130, 1040, 4008), (3, 270, 390, 1365)], ids=str)
def test_long_sums(nn, dtype, size):
    """Sizes at which a product's k is shared out among wavefronts, with more tiles than CUs where those are small."""
    t = tensors(*size, dtype, seed=16)
    _, got = train(nn, t, dtype, "silu")
    check("silu", dtype, t, got, NAMES)


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
def test_strides_and_alignment(nn, dtype):
    """Rows further apart than they are long, workers next to each other, tensors that begin anywhere; what lies between is NaN and is not touched."""
    W, T, D, F = 2, 37, 72, 88
    t = tensors(W, T, D, F, dtype, seed=3)

    def spread(v, lead, gap):
        w, r, c = v.shape
        flat = torch.full((lead + w * r * (c + gap),), float("nan"), dtype=dtype, device="cuda")
        view = flat[lead:].view(w, r, c + gap)[:, :, :c]
        view.copy_(v)
        return flat, view

    for lead, gap in ((0, 8), (8, 24), (1, 1), (3, 5)):
        s = {k: spread(v, lead, gap) for k, v in t.items()}
        op = nn.GatedFFN(D, F, workers=W, max_rows=T, dtype=dtype, train=True)
        outs = {k: spread(torch.zeros_like(t[o]), lead, gap) for k, o in (("y", "x"), ("dx", "x"), ("dw_gate", "w_gate"), ("dw_up", "w_up"), ("dw_down", "w_down"))}
        view = {k: v[1] for k, v in s.items()}
        _, saved = op.forward(view["x"], view["w_gate"], view["w_up"], view["w_down"], out=outs["y"][1], save=True)
        op.backward(view["dy"], view["x"], view["w_gate"], view["w_up"], view["w_down"], saved,
                    **{k: outs[k][1] for k in ("dx", "dw_gate", "dw_up", "dw_down")})
        check("silu", dtype, t, {k: v[1] for k, v in outs.items()}, NAMES)
        for k, (flat, v) in outs.items():
            kept = flat.clone()
            kept[lead:].view(W, v.shape[1], -1)[:, :, :v.shape[2]] = float("nan")
            assert torch.isnan(kept).all(), k


def test_workers_side_by_side(nn):
    """Workers as the second axis of memory, and one weight that all workers share (stride 0)."""
    t = tensors(3, 20, 64, 96, torch.bfloat16, seed=4)
    x = t["x"].transpose(0, 1).contiguous().transpose(0, 1)
    shared = {k: t[k][:1].expand(3, -1, -1) for k in ("w_gate", "w_up", "w_down")}
    op = nn.GatedFFN(64, 96, workers=3, max_rows=20)
    out = torch.empty(20, 3, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    op.forward(x, shared["w_gate"], shared["w_up"], shared["w_down"], out=out)
    check("silu", torch.bfloat16, dict(t, **shared), dict(y=out), ("y",))


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("size", [(2, 70, 72, 136), (1, 90, 65, 33), (1, 9, 64, 64)], ids=str)
def test_broadcast_tokens(nn, dtype, size):
    """One row of memory for all tokens, as a gradient of a sum over them has; rows that lie closer than they are long."""
    W, T, D, F = size
    t = tensors(*size, dtype, seed=13)
    for k in ("x", "dy"):
        t[k] = t[k][:, :1].expand(W, T, D)
    _, got = train(nn, t, dtype, "silu")
    check("silu", dtype, t, got, NAMES)
    flat = torch.randn(W, 8 * T + D, generator=torch.Generator().manual_seed(14)).to(dtype).cuda()
    t = dict(tensors(*size, dtype, seed=15), x=flat.as_strided((W, T, D), (flat.shape[1], 8, 1)))
    _, got = train(nn, t, dtype, "silu")
    check("silu", dtype, t, got, NAMES)


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
def test_no_tokens(nn, dtype):
    t = tensors(2, 0, 24, 40, dtype)
    _, got = train(nn, t, dtype, "silu")
    assert got["y"].shape == (2, 0, 24) and got["dx"].shape == (2, 0, 24)
    assert all(float(got[k].abs().max()) == 0.0 for k in ("dw_gate", "dw_up", "dw_down"))


def test_only_some_gradients(nn):
    t = tensors(1, 30, 64, 64, torch.float16, seed=5)
    op, got = train(nn, t, torch.float16, "silu", input_gradient=False)
    assert got["dx"] is None
    check("silu", torch.float16, t, got, ("y", "dw_gate", "dw_up", "dw_down"))


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
def test_large_arguments_of_the_activation(nn, dtype):
    """Projections far out on both sides: the activation neither overflows nor becomes NaN."""
    t = tensors(1, 8, 64, 64, dtype, seed=6)
    t["w_gate"] *= 200
    for kind in ("silu", "gelu", "gelu_tanh", "relu"):
        _, got = train(nn, t, dtype, kind)
        check(kind, dtype, t, got, NAMES)


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
def test_what_is_not_finite_stays_with_its_token(nn, dtype):
    t = tensors(1, 70, 64, 72, dtype, seed=7)
    t["x"][0, 5, 3] = float("nan")
    t["x"][0, 66, 1] = float("inf")
    _, got = train(nn, t, dtype, "silu")
    bad = torch.zeros(70, dtype=torch.bool, device="cuda")
    bad[[5, 66]] = True
    assert torch.isfinite(got["y"][0][~bad]).all() and torch.isfinite(got["dx"][0][~bad]).all()
    assert not torch.isfinite(got["y"][0][bad]).any() and torch.isnan(got["dw_gate"][0]).any()


def test_offsets_beyond_32_bits(nn):
    """Tokens whose elements lie beyond 2^31, and rows 2^25 elements apart."""
    T, D, F = 1_100_001, 2048, 64
    gen = torch.Generator(device="cuda").manual_seed(11)
    make = lambda *s, size=1.0: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(generator=gen).mul_(size)
    t = dict(x=make(1, T, D), w_gate=make(1, F, D, size=D ** -0.5), w_up=make(1, F, D, size=D ** -0.5), w_down=make(1, D, F, size=F ** -0.5), dy=make(1, T, D))
    _, got = train(nn, t, torch.bfloat16, "silu")
    ends = torch.cat([torch.arange(40), torch.arange(T - 300, T)]).cuda()
    some = {k: (v[:, ends] if k in ("x", "dy") else v) for k, v in t.items()}
    check("silu", torch.bfloat16, some, dict(y=got["y"][:, ends], dx=got["dx"][:, ends]), ("y", "dx"), device="cuda")
    want = {k: 0.0 for k in NAMES[2:]}
    for a in range(0, T, 100_000):
        v = {k: (x[0, a:a + 100_000] if k in ("x", "dy") else x[0]).double() for k, x in t.items()}
        part = ref.ffn("silu", torch.bfloat16, v["x"], v["w_gate"], v["w_up"], v["w_down"], v["dy"])
        want = {k: want[k] + part[k][0] for k in want}
    for k in want:
        # dg, du and h are rounded, then the sums: each at most a unit off, independently; a million additions in 32 bits stay far below
        off = float((got[k][0].double() - want[k]).norm() / want[k].norm())
        print(f"[ffn] {k} of {T} tokens: {off / ref.UNIT[torch.bfloat16]:.2f} units", flush=True)
        assert off <= 4 * ref.UNIT[torch.bfloat16], k
    del t, got, some
    torch.cuda.empty_cache()
    t = tensors(1, 70, 64, 96, torch.bfloat16, seed=12)
    far = torch.empty(69 * 2 ** 25 + 64, dtype=torch.bfloat16, device="cuda")
    x = far.as_strided((1, 70, 64), (far.numel(), 2 ** 25, 1))
    x.copy_(t["x"])
    op = nn.GatedFFN(64, 96, max_rows=70)
    check("silu", torch.bfloat16, t, dict(y=op.forward(x, t["w_gate"], t["w_up"], t["w_down"])), ("y",))


def test_same_bits_every_time_and_in_a_graph(nn):
    t = tensors(2, 130, 256, 320, torch.bfloat16, seed=8)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        op = nn.GatedFFN(256, 320, workers=2, max_rows=130, train=True, stream=stream)

        def once():
            y, saved = op.forward(t["x"], t["w_gate"], t["w_up"], t["w_down"], save=True)
            return (y, *op.backward(t["dy"], t["x"], t["w_gate"], t["w_up"], t["w_down"], saved))

        torch.cuda.synchronize()
        first = [v.clone() for v in once()]
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            kept = once()
        for _ in range(3):
            for v in kept:
                v.fill_(7.0)
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(first, kept))
            again = once()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_gradient_against_differences(nn):
    """Along a random direction in each input, the 32-bit gradient against central differences of the block in 64 bits."""
    W, T, D, F = 1, 19, 40, 56
    for kind in ("silu", "gelu", "gelu_tanh"):
        t = tensors(W, T, D, F, torch.float32, seed=9)
        _, got = train(nn, t, torch.float32, kind)
        v = {k: t[k][0].cpu().double() for k in t}
        loss = lambda x, wg, wu, wd: float(((ref.act(kind, x @ wg.t())[0] * (x @ wu.t())) @ wd.t() * v["dy"]).sum())
        names = ("x", "w_gate", "w_up", "w_down")
        gen = torch.Generator().manual_seed(10)
        for i, name in enumerate(names):
            d = torch.randn(v[name].shape, generator=gen, dtype=torch.float64)
            step = 1e-5
            args = [[v[n] + (s * step * d if n == name else 0) for n in names] for s in (1, -1)]
            slope = (loss(*args[0]) - loss(*args[1])) / (2 * step)
            mine = float((got["d" + name][0].cpu().double() * d).sum())
            size = float((got["d" + name][0].cpu().double().abs() * d.abs()).sum())
            # differences: third derivative times step^2, and 2^-52 / step of the loss; the gradient: its bound of some 2000 U32
            assert abs(slope - mine) <= 1e-5 * size, (kind, name, slope, mine)


def test_refusals(nn):
    from paper_2103_07454_amd import evg
    t = tensors(1, 8, 64, 64, torch.bfloat16)
    op = nn.GatedFFN(64, 64, max_rows=8)
    args = (t["x"], t["w_gate"], t["w_up"], t["w_down"])
    for bad in ((t["x"].float(), *args[1:]), (t["x"].cpu(), *args[1:]), (t["x"][:, :, :32], *args[1:]), (t["x"][0], *args[1:]),
                (t["x"].repeat(1, 2, 1), *args[1:]), (args[0], t["w_gate"][:, :32], *args[2:]),
                (args[0], args[1], args[2], t["w_down"].transpose(1, 2))):
        with pytest.raises(ValueError):
            op.forward(*bad)
    with pytest.raises(evg.EvgError):
        op.forward(*args, out=t["x"])                                    # the output on an input
    with pytest.raises(evg.EvgError):
        op.forward(*args, out=torch.empty(1, 1, 64, dtype=torch.bfloat16, device="cuda").expand(1, 8, 64))   # rows that overlap
    y, saved = op.forward(*args, save=True)
    with pytest.raises(evg.EvgError) as e:
        op.backward(t["dy"], *args, saved)                               # made without train
    assert e.value.status == 5
    trained = nn.GatedFFN(64, 64, max_rows=8, train=True)
    with pytest.raises(ValueError):
        trained.backward(t["dy"], *args, saved[:-16])
    with pytest.raises(evg.EvgError):
        trained.backward(t["dy"], *args, saved, dw_gate=t["w_gate"])
    for bad in (dict(width=0), dict(hidden=0), dict(workers=0), dict(activation=9), dict(max_rows=0x7FFFFFFF, workers=65535)):
        with pytest.raises(evg.EvgError):
            nn.GatedFFN(**{**dict(width=64, hidden=64, max_rows=8), **bad})
    with pytest.raises(ValueError):
        nn.GatedFFN(64, 64, max_rows=8, dtype=torch.float64)
