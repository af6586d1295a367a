"""The norms around a block against their definition in 64 bits (tests/nn_reference.py), and their refusals."""
import itertools

import pytest
import torch

import nn_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
SHORT = {torch.bfloat16: "bf16", torch.float16: "f16", torch.float32: "f32"}
ALPHA, BETA, EPS = 0.9, 1.25, 1e-5


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


def tensors(W, T, D, dtype, kind, gate_rows, *, branch=True, post=True, pre=True, bias=True, seed=0):
    gen = torch.Generator().manual_seed(seed)
    make = lambda *s, size=1.0, mean=0.0: (torch.randn(*s, generator=gen) * size + mean).to(dtype).cuda()
    t = dict(residual=make(W, T, D, size=2.0))
    if branch:
        t["branch"] = make(W, T, D, size=0.7, mean=0.1)
        if gate_rows:
            t["gate"] = make(W, -(-T // gate_rows), D, size=0.5, mean=0.5)
        if post:
            t["post"] = make(W, D, size=0.2, mean=0.5)
            if kind == "layer" and bias:
                t["post_bias"] = make(W, D, size=0.2)
    if pre:
        t["pre"] = make(W, D, size=0.2, mean=1.0)
        if kind == "layer" and bias:
            t["pre_bias"] = make(W, D, size=0.2)
    return t, make(W, T, D), make(W, T, D)


def limits(want, size, terms, dtype):
    """Elementwise bound.  Values pass through some ten operations and at most two sums over the row (32 bits, partial sums of at most
    16 terms in a lane and 10 levels above: 26 roundings), each off by so many units of 2^-24 of the terms' magnitudes, which `size` has
    from the reference, before they cancel: 128 units hold both.  Sums over `terms` rows add terms' roundings: 4 sqrt(terms)
    times as many at most of the terms' root sum of squares."""
    scale = size.square().mean(-1, keepdim=True).sqrt() + size
    return 128 * ref.U32 * scale * (1 + 4 * terms ** 0.5) + ref.rounding(want, dtype) * 1.001


def check(nn, kind, dtype, t, d_out, d_normed, gate_rows, backward=True, op=None):
    W, T, D = t["residual"].shape
    op = op or nn.BlockNorm(D, workers=W, max_rows=T, dtype=dtype, kind=nn.LAYER if kind == "layer" else nn.RMS, eps=EPS,
                            residual_scale=ALPHA, branch_scale=BETA, gate_rows=gate_rows)
    given = {k: t.get(k) for k in ("branch", "gate", "post", "post_bias", "pre", "pre_bias")}
    r, n = op.forward(t["residual"], **given)
    got = dict(residual=r)
    if n is not None:
        got["normed"] = n
    if backward:
        got.update(op.backward(d_out, d_normed if "pre" in t else None, t["residual"], **given))
    worst = {}
    for w in range(W):
        v = {k: x[w].cpu().double() for k, x in t.items()}
        if backward:
            if d_out is not None:
                v["d_out"] = d_out[w].cpu().double()
            if d_normed is not None and "pre" in t:
                v["d_normed"] = d_normed[w].cpu().double()
        want, size = ref.blocknorm(kind, v, eps=EPS, alpha=ALPHA, beta=BETA, gate_rows=gate_rows)
        assert set(got) == set(want) or not backward
        for name, g in got.items():
            terms = T if name in ("d_pre", "d_post", "d_pre_bias", "d_post_bias") else min(gate_rows, T) if name == "d_gate" else 0
            assert torch.isfinite(g[w]).all(), name
            off = (g[w].cpu().double() - want[name]).abs() / limits(want[name], size[name], terms, dtype)
            worst[name] = max(worst.get(name, 0.0), float(off.max()) if off.numel() else 0.0)
    print(f"\n[norm] {SHORT[dtype]} {kind} {(W, T, D)} gate_rows {gate_rows}: share of the bound "
          + ", ".join(f"{k} {v:.2g}" for k, v in worst.items()), flush=True)
    assert all(v <= 1.0 for v in worst.values()), worst
    return got


# widths on both sides of 8, 64, and of what 64, 128, 256, 512 and 1024 threads hold; one row, odd numbers of rows
SIZES = [(1, 1, 1024), (1, 1, 2), (2, 3, 7), (1, 5, 64), (3, 9, 511), (1, 4, 513), (2, 33, 1000), (1, 7, 1025), (1, 130, 2048), (1, 3, 2056),
         (1, 17, 4095), (1, 2, 4100), (1, 3, 8192), (2, 2, 8200), (1, 3, 16384), (1, 2100, 65)]


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(nn, dtype, kind, size):
    t, d_out, d_normed = tensors(*size, dtype, kind, 2)
    check(nn, kind, dtype, t, d_out, d_normed, 2)


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("size", [(1, 3, 8), (1, 17, 127), (2, 15, 128), (1, 33, 129), (3, 7, 255), (1, 9, 256), (1, 5, 257), (2, 2500, 33), (1, 4100, 130)], ids=str)
def test_narrow_rows(nn, dtype, kind, size):
    """Widths around what 16 and 32 threads hold; rows that fill a workgroup and do not; more rows than stripes."""
    t, d_out, d_normed = tensors(*size, dtype, kind, 3, seed=6)
    check(nn, kind, dtype, t, d_out, d_normed, 3)


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
@pytest.mark.parametrize("rows,gate_rows", [(1, 1), (9, 1), (9, 4), (9, 9), (9, 100), (2500, 1), (2500, 2), (2500, 3), (2500, 7), (2500, 1000),
                                            (2500, 2500), (1025, 1024)])
def test_gates(nn, dtype, rows, gate_rows):
    t, d_out, d_normed = tensors(2, rows, 72, dtype, "rms", gate_rows, seed=1)
    check(nn, "rms", dtype, t, d_out, d_normed, gate_rows)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("branch,post,pre,gate,bias", [c for c in itertools.product((0, 1), repeat=5) if c[0] or not (c[1] or c[3])])
def test_what_may_be_absent(nn, kind, branch, post, pre, gate, bias):
    gate_rows = 5 if gate else 0
    t, d_out, d_normed = tensors(2, 12, 136, torch.float32, kind, gate_rows, branch=branch, post=post, pre=pre, bias=bias, seed=2)
    check(nn, kind, torch.float32, t, d_out, d_normed, gate_rows)
    if pre:
        check(nn, kind, torch.float32, t, None, d_normed, gate_rows)
        check(nn, kind, torch.float32, t, d_out, None, gate_rows)


def test_many_workers(nn):
    t, d_out, d_normed = tensors(1500, 2, 40, torch.float32, "layer", 2, seed=3)
    op = nn.BlockNorm(40, workers=1500, max_rows=2, dtype=torch.float32, kind=nn.LAYER, eps=EPS, residual_scale=ALPHA,
                      branch_scale=BETA, gate_rows=2)
    check(nn, "layer", torch.float32, t, d_out, d_normed, 2, op=op)


@pytest.mark.parametrize("dtype", TYPES, ids=SHORT.get)
def test_strides_and_alignment(nn, dtype):
    """Rows anywhere, what lies between them NaN and untouched; the residual updated in place."""
    W, T, D = 2, 21, 136
    t, d_out, d_normed = tensors(W, T, D, dtype, "layer", 4, seed=4)
    plain = check(nn, "layer", dtype, t, d_out, d_normed, 4)

    def spread(v, lead, gap):
        rows = v.shape[1] if v.dim() == 3 else 1
        flat = torch.full((lead + W * rows * (D + gap),), float("nan"), dtype=dtype, device="cuda")
        view = flat[lead:].view(W, rows, D + gap)[:, :, :D]
        view = view if v.dim() == 3 else view[:, 0]
        view.copy_(v)
        return flat, view

    for lead, gap in ((8, 24), (1, 1), (3, 5)):
        s = {k: spread(v, lead, gap)[1] for k, v in t.items()}
        op = nn.BlockNorm(D, workers=W, max_rows=T, dtype=dtype, kind=nn.LAYER, eps=EPS, residual_scale=ALPHA, branch_scale=BETA, gate_rows=4)
        given = {k: v for k, v in s.items() if k != "residual"}
        outs = {k: spread(torch.zeros_like(v), lead, gap) for k, v in plain.items()}
        op.forward(s["residual"], residual_out=outs["residual"][1], normed=outs["normed"][1], **given)
        op.backward(spread(d_out, lead, gap)[1], spread(d_normed, lead, gap)[1], s["residual"], out={k: v[1] for k, v in outs.items()}, **given)
        for k, (flat, v) in outs.items():
            assert torch.equal(v, plain[k]), k
            v.fill_(float("nan"))
            assert torch.isnan(flat).all(), k
        r, n = op.forward(s["residual"], residual_out=s["residual"], **given)
        assert r is s["residual"] and torch.equal(r, plain["residual"]) and torch.equal(n, plain["normed"])


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_no_rows(nn, kind):
    t, d_out, d_normed = tensors(2, 0, 64, torch.float32, kind, 4)
    got = check(nn, kind, torch.float32, t, d_out, d_normed, 4)
    assert got["d_gate"].shape == (2, 0, 64) and all(float(got[k].abs().max()) == 0.0 for k in ("d_pre", "d_post"))


def test_rows_of_zeros_and_large_values(nn):
    """A row of zeros has the unit row 0; squares are not rounded to 16 bits on the way, so values near a type's end are fine."""
    for dtype, big in ((torch.float16, 3e4), (torch.bfloat16, 1e15), (torch.float32, 1e15)):
        op = nn.BlockNorm(300, max_rows=3, dtype=dtype, eps=EPS)
        x = torch.zeros(1, 3, 300, dtype=dtype, device="cuda")
        x[0, 1] = big
        w = torch.ones(1, 300, dtype=dtype, device="cuda")
        r, n = op.forward(x, pre=w)
        assert r is x
        assert float(n[0, 0].abs().max()) == 0.0 and float(n[0, 2].abs().max()) == 0.0
        assert float((n[0, 1] - 1).abs().max()) <= 2 * ref.UNIT[dtype]
    layer = nn.BlockNorm(300, max_rows=1, dtype=torch.float32, kind=nn.LAYER, eps=EPS)
    x = torch.full((1, 1, 300), 1e4, device="cuda")         # constant rows: no variance
    _, n = layer.forward(x, pre=torch.ones(1, 300, device="cuda"), pre_bias=torch.full((1, 300), 0.25, device="cuda"))
    # the mean of 300 equal values is off by a few units of 2^-24: 1e4 * 2^-22 / sqrt(eps) at most
    assert float((n - 0.25).abs().max()) <= 1e4 * 2.0 ** -22 / EPS ** 0.5


def test_what_is_not_finite_stays_in_its_row(nn):
    t, d_out, d_normed = tensors(1, 9, 200, torch.float32, "rms", 0, seed=5)
    t["residual"][0, 3, 7] = float("nan")
    t["branch"][0, 5, 9] = float("inf")
    op = nn.BlockNorm(200, max_rows=9, dtype=torch.float32, eps=EPS)
    r, n = op.forward(t["residual"], t["branch"], post=t["post"], pre=t["pre"])
    ok = [0, 1, 2, 4, 6, 7, 8]
    assert torch.isfinite(n[0, ok]).all() and not torch.isfinite(n[0, 3]).any() and torch.isnan(n[0, 5]).any()
    d = op.backward(d_out, d_normed, t["residual"], t["branch"], post=t["post"], pre=t["pre"])
    assert torch.isfinite(d["d_residual"][0, ok]).all() and torch.isfinite(d["d_branch"][0, ok]).all()


def test_offsets_beyond_32_bits(nn):
    T, D = 1_100_001, 2048
    gen = torch.Generator(device="cuda").manual_seed(9)
    make = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    t = dict(residual=make(1, T, D), branch=make(1, T, D), pre=make(1, D), post=make(1, D))
    d_out, d_normed = make(1, T, D), make(1, T, D)
    op = nn.BlockNorm(D, max_rows=T, eps=EPS)
    given = {k: v for k, v in t.items() if k != "residual"}
    r, n = op.forward(t["residual"], **given)
    d = op.backward(d_out, d_normed, t["residual"], **given)
    ends = torch.cat([torch.arange(40), torch.arange(T - 300, T)]).cuda()
    v = {k: (x[0, ends] if x.dim() == 3 else x[0]).cpu().double() for k, x in t.items()}
    v.update(d_out=d_out[0, ends].cpu().double(), d_normed=d_normed[0, ends].cpu().double())
    want, size = ref.blocknorm("rms", v, eps=EPS, alpha=1.0, beta=1.0, gate_rows=1)
    for name, g in (("residual", r), ("normed", n), ("d_residual", d["d_residual"]), ("d_branch", d["d_branch"])):
        off = (g[0, ends].cpu().double() - want[name]).abs()
        assert bool((off <= limits(want[name], size[name], 0, torch.bfloat16)).all()), name
    total = torch.zeros(D, dtype=torch.float64, device="cuda")
    for a in range(0, T, 100_000):
        rr = t["residual"][0, a:a + 100_000].double() + ref.unit("rms", t["branch"][0, a:a + 100_000].double(), EPS)[0] * t["post"][0].double()
        total += (d_normed[0, a:a + 100_000].double() * ref.unit("rms", rr, EPS)[0]).sum(0)
    # independent terms of size 1: the bound of a sum over T rows, and the rounding
    off = (d["d_pre"][0].double() - total).abs()
    assert bool((off <= 128 * ref.U32 * T ** 0.5 * (1 + 4 * T ** 0.5) + ref.rounding(total, torch.bfloat16) * 1.001).all())


def test_same_bits_every_time_and_in_a_graph(nn):
    t, d_out, d_normed = tensors(1, 3000, 520, torch.bfloat16, "rms", 1000, seed=6)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        op = nn.BlockNorm(520, max_rows=3000, eps=EPS, gate_rows=1000, stream=stream)
        given = {k: v for k, v in t.items() if k != "residual"}

        def once():
            return (*op.forward(t["residual"], **given), *op.backward(d_out, d_normed, t["residual"], **given).values())

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


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradient_against_differences(nn, kind):
    t, d_out, d_normed = tensors(1, 11, 48, torch.float32, kind, 4, seed=7)
    got = check(nn, kind, torch.float32, t, d_out, d_normed, 4)
    v = {k: x[0].cpu().double() for k, x in t.items()}
    do, dn = d_out[0].cpu().double(), d_normed[0].cpu().double()

    def loss(u):
        o, _ = ref.blocknorm(kind, u, eps=EPS, alpha=ALPHA, beta=BETA, gate_rows=4)
        return float((o["residual"] * do).sum() + (o["normed"] * dn).sum())

    gen = torch.Generator().manual_seed(8)
    for name in v:
        d = torch.randn(v[name].shape, generator=gen, dtype=torch.float64)
        step = 1e-5
        slope = (loss({**v, name: v[name] + step * d}) - loss({**v, name: v[name] - step * d})) / (2 * step)
        g = got["d_" + name][0].cpu().double()
        # the differences: step^2 of a third derivative, 2^-52 / step of the loss; the gradient: 128 units of 2^-24 and some
        assert abs(slope - float((g * d).sum())) <= 3e-5 * float((g.abs() * d.abs()).sum()), (name, slope)


def test_refusals(nn):
    from paper_2103_07454_amd import evg
    t, d_out, d_normed = tensors(1, 8, 64, torch.bfloat16, "rms", 2)
    op = nn.BlockNorm(64, max_rows=8, gate_rows=2)
    given = {k: v for k, v in t.items() if k != "residual"}
    r = t["residual"]
    for bad in (dict(branch=r.float()), dict(branch=r[:, :4]), dict(gate=r), dict(pre=r[0, 0]), dict(post=t["post"].cpu())):
        with pytest.raises(ValueError):
            op.forward(r, **{**given, **bad})
    for bad in (r.repeat(1, 2, 1), r[0]):
        with pytest.raises(ValueError):
            op.forward(bad, **given)
    with pytest.raises(ValueError):
        nn.BlockNorm(64, max_rows=8).forward(r, **given)                   # a gate without gate_rows
    for bad in (dict(branch=None), dict(branch=None, gate=None), dict(pre_bias=t["pre"]), dict(pre=None, pre_bias=t["pre"]),
                dict(residual_out=t["branch"]), dict(normed=r), dict(pre=None, normed=torch.empty_like(r))):
        with pytest.raises(evg.EvgError):
            op.forward(r, **{**given, **bad})
    with pytest.raises(evg.EvgError):
        op.backward(d_out, d_normed, r, out=dict(d_branch=t["branch"]), **given)
    with pytest.raises(evg.EvgError):
        op.backward(d_out, d_normed, r, **{**given, "pre": None})
    for bad in (dict(width=0), dict(width=16385), dict(workers=0), dict(kind=2), dict(eps=-1.0), dict(eps=float("nan")),
                dict(residual_scale=float("inf"))):
        with pytest.raises(evg.EvgError):
            nn.BlockNorm(**{**dict(width=64, max_rows=8), **bad})
