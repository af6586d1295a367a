"""What a user of this framework has its operators for training feed-forward blocks do, as cases that can be timed.

Three operators belong together: each ring worker normalises what its block reads and adds the block's output to its
residual stream through a gate (`nn.BlockNorm`), runs its gated feed-forward block and that block's backward pass
(`nn.GatedFFN`), and bounds the global norm of its gradient before the ring's step takes it (`nn.GradClip`). All workers
of a ring go in one call: tensors have the worker as their first axis.

With W workers, T tokens of each, a width D and a hidden width F, for each worker:

    clip    norm = scale * sqrt(sum of g^2 over all its tensors),  out = g * scale * min(1, max_norm / (norm + 1e-6))
    norm    r' = a * r + b * gate * N(branch; post),  n = N(r'; pre),  N the RMS or the layer norm over D
    ffn     y = (act(x Wg^T) * (x Wu^T)) Wd^T

and the gradients of the latter two with respect to every tensor that they read.
"""
import math

import torch

own = False

_TYPE = dict(f32=torch.float32, f16=torch.float16, bf16=torch.bfloat16)
_SIZE = dict(f32=4, f16=2, bf16=2)
#: Elements of the largest listed clipped gradient, operations of the largest feed-forward block, values of the largest norm.
MOST_CLIPPED = 64 * 11_173_962
MOST_FLOPS = 18 * 8192 * 2048 * 8192
MOST_NORMED = 16384 * 4096


def _clip(name, net, width, workers, dtype, out, scale=1.0):
    return dict(name=name, op="clip", net=net, width=width, workers=workers, dtype=dtype, out=out, scale=scale)


def _norm(name, workers, tokens, width, dtype, kind, post, gate_rows, train):
    return dict(name=name, op="norm", workers=workers, tokens=tokens, width=width, dtype=dtype, kind=kind, post=post,
                gate_rows=gate_rows, train=train)


def _ffn(name, workers, tokens, width, hidden, dtype, activation, train):
    return dict(name=name, op="ffn", workers=workers, tokens=tokens, width=width, hidden=hidden, dtype=dtype,
                activation=activation, train=train)


def listed():
    return [
        # the smallest ring that is trained, a two-layer perceptron on four workers: what an iteration pays at least
        _clip("clip_mlp_p4", "mlp", 128, 4, "f32", "f32"),
        # 62 ragged tensors of seven workers, gradients in half the bits with a loss scale, clipped into the ring's arena
        _clip("clip_resnet18w23_p7_bf16", "resnet18", 23, 7, "bf16", "f32", scale=1.0 / 1024),
        # the headline benchmark's ring: 715 million elements
        _clip("clip_resnet18_p64", "resnet18", 64, 64, "f32", "f32"),
        # one new token of one model: the norm before its next block, on top of the last block's output
        _norm("norm_token", 1, 1, 1024, "bf16", "rms", False, 0, False),
        # a prompt through norms on both sides of a block with a gate for every value
        _norm("norm_prompt_f16", 1, 2049, 2048, "f16", "rms", True, 1, False),
        # eight small workers trained in 32 bits, layer norms, one gate for all tokens of a worker; odd in every size
        _norm("norm_ring_layer_f32", 8, 333, 785, "f32", "layer", True, 333, True),
        # a long training batch: norms on both sides, a gate for each sequence of 2048 tokens
        _norm("norm_train", 1, 16384, 4096, "bf16", "rms", True, 2048, True),
        # one new token through a feed-forward block: the weights are read once
        _ffn("ffn_token", 1, 1, 2048, 5632, "bf16", "silu", False),
        # a prompt
        _ffn("ffn_prompt", 1, 4096, 4096, 11264, "bf16", "silu", False),
        # eight workers' small blocks trained at once, an odd hidden width
        _ffn("ffn_ring_f16", 8, 250, 512, 1365, "f16", "gelu_tanh", True),
        # four workers in 32 bits, as the ring holds its parameters: the perceptron's widths
        _ffn("ffn_ring_f32", 4, 100, 784, 203, "f32", "gelu", True),
        # a training batch, forward and backward: every gradient
        _ffn("ffn_train", 1, 8192, 2048, 8192, "bf16", "silu", True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _width(rng, lo, hi):
    """Widths are mostly whole cache lines; one in three is any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 1 / 3 else max(lo, n // 64 * 64)


def draw(rng):
    """One of the operators over the range of its listed cases: rings of 1 to 64 workers, one token to long batches, narrow
    widths to wide ones, any number between."""
    while True:
        op = rng.choice(("clip", "norm", "ffn"))
        if op == "clip":
            net = rng.choice(("mlp", "resnet18", "block"))
            width = {"mlp": lambda: _log_int(rng, 32, 1024), "resnet18": lambda: _log_int(rng, 8, 64),
                     "block": lambda: _width(rng, 64, 2048)}[net]()
            dtype = rng.choice(("f32", "f32", "bf16", "f16"))
            case = _clip("", net, width, _log_int(rng, 1, 64), dtype, rng.choice(("f32", dtype)), rng.choice((1.0, 1.0 / 1024)))
            fits = case["workers"] * sum(_numel(case)) <= MOST_CLIPPED
        elif op == "norm":
            tokens = _log_int(rng, 1, 16384)
            case = _norm("", _log_int(rng, 1, 16), tokens, _width(rng, 64, 8192), rng.choice(("bf16", "f16", "f32")),
                         rng.choice(("rms", "rms", "layer")), rng.random() < 0.6,
                         rng.choice((0, 1, tokens, _log_int(rng, 1, tokens))), rng.random() < 0.6)
            fits = case["workers"] * tokens * case["width"] * _SIZE[case["dtype"]] <= 2 * MOST_NORMED
        else:
            case = _ffn("", rng.choice((1, 1, 1, _log_int(rng, 2, 16))), _log_int(rng, 1, 8192), _width(rng, 64, 4096),
                        _width(rng, 64, 11264), rng.choice(("bf16", "bf16", "f16", "f32")),
                        rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu")), rng.random() < 0.5)
            # 32-bit products go at a sixteenth of the rate
            fits = work(case)["flops"] * (16 if case["dtype"] == "f32" else 1) <= MOST_FLOPS
        if fits and 3 << 10 not in case.values():
            del case["name"]
            return case


def _numel(case):
    """The lengths of one worker's tensors."""
    w = case["width"]
    if case["net"] == "mlp":
        return [784 * w, w, w * 10, 10]
    if case["net"] == "block":  # two feed-forward blocks, each with the norms on its sides
        return [w, 4 * w * w, 4 * w * w, 4 * w * w, w] * 2
    sizes = [27 * w, w, w]
    c_in = w
    for stage in range(4):
        c = w << stage
        for block in range(2):
            sizes += [9 * c_in * c, c, c, 9 * c * c, c, c]
            if stage and not block:
                sizes += [c_in * c, c, c]
            c_in = c
    return sizes + [8 * w * 10, 10]


def _places(case):
    """Where a worker's tensors begin in its slice of an arena, and the slice's length: starts are padded to 4, the slice to 64."""
    at, starts = 0, []
    for n in _numel(case):
        starts.append(at)
        at += (n + 3) // 4 * 4
    return starts, (at + 63) // 64 * 64


def work(case):
    e = _SIZE[case["dtype"]]
    if case["op"] == "clip":
        n = case["workers"] * sum(_numel(case))
        return {"bytes": float(n * (e + _SIZE[case["out"]])), "flops": 3.0 * n}
    rows = case["workers"] * case["tokens"]
    d = case["width"]
    if case["op"] == "norm":
        gates = 0 if not case["gate_rows"] else case["workers"] * -(-case["tokens"] // case["gate_rows"]) * d
        weights = case["workers"] * d * (1 + case["post"]) * (1 + (case["kind"] == "layer"))
        values = 4 * rows * d + gates + weights
        flops = 12.0 * rows * d
        if case["train"]:  # what the forward pass read is read again only if it does not stay at hand
            values += 4 * rows * d + gates + weights
            flops += 30.0 * rows * d
        return {"bytes": float(e * values), "flops": flops}
    f = case["hidden"]
    weights = 3 * case["workers"] * d * f
    return {"bytes": float(e * (2 * rows * d + weights) * (2 if case["train"] else 1)),
            "flops": (18.0 if case["train"] else 6.0) * rows * d * f}


def _inputs(case, seed):
    """Tensors of the case on the GPU, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, workers = _TYPE[case["dtype"]], case["workers"]

    def normal(*shape, size=1.0, mean=0.0):
        t = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)
        return t.mul_(size).add_(mean) if mean else t.mul_(size)

    if case["op"] == "clip":
        numel, (starts, pitch) = _numel(case), _places(case)
        grad = normal(workers, pitch)  # what lies between the tensors is anything
        real = torch.zeros(pitch, dtype=torch.bool, device="cuda")
        rows = torch.randn(workers, generator=gen, device="cuda").exp_()  # some workers' gradients are long, some short
        for at, n in zip(starts, numel):
            real[at:at + n] = True
        size = 1e-2 if case["scale"] == 1.0 else 1e-2 * 1024
        grad.mul_((rows * size)[:, None].to(dtype))
        return dict(grad=grad, real=real, out=torch.zeros(workers, pitch, dtype=_TYPE[case["out"]], device="cuda"),
                    max_norm=1e-2 * math.sqrt(sum(numel)))
    tokens, d = case["tokens"], case["width"]
    if case["op"] == "norm":
        t = dict(residual=normal(workers, tokens, d, size=2.0), branch=normal(workers, tokens, d, size=0.7),
                 pre=normal(workers, d, size=0.2, mean=1.0))
        t["residual"][..., ::97] *= 8  # a few wide channels, as residual streams have
        if case["gate_rows"]:
            t["gate"] = normal(workers, -(-tokens // case["gate_rows"]), d, size=0.5, mean=0.5)
        if case["post"]:
            t["post"] = normal(workers, d, size=0.2, mean=0.5)
        if case["kind"] == "layer":
            t["pre_bias"] = normal(workers, d, size=0.2)
            if case["post"]:
                t["post_bias"] = normal(workers, d, size=0.2)
        if case["train"]:
            t["d_residual"], t["d_normed"] = normal(workers, tokens, d), normal(workers, tokens, d)
        return t
    f = case["hidden"]
    t = dict(x=normal(workers, tokens, d), w_gate=normal(workers, f, d, size=d ** -0.5),
             w_up=normal(workers, f, d, size=d ** -0.5), w_down=normal(workers, d, f, size=f ** -0.5))
    if case["train"]:
        t["dy"] = normal(workers, tokens, d)
    return t


#: What the norm's cases scale the residual and the branch by, and the constant under its root.
RESIDUAL, BRANCH, EPS = 0.9, 1.25, 1e-5


def prepare(case, seed):
    """The tensors that a pass reads, and the operator's handle where it has one."""
    state = dict(case=case, t=_inputs(case, seed))
    if own:
        from paper_2103_07454_amd import nn
        dtype = _TYPE[case["dtype"]]
        if case["op"] == "clip":
            state["op"] = nn.GradClip(_numel(case), case["workers"], dtype=dtype, out_dtype=_TYPE[case["out"]])
        elif case["op"] == "norm":
            state["op"] = nn.BlockNorm(case["width"], workers=case["workers"], max_rows=case["tokens"], dtype=dtype,
                                       kind=nn.LAYER if case["kind"] == "layer" else nn.RMS, eps=EPS, residual_scale=RESIDUAL,
                                       branch_scale=BRANCH, gate_rows=case["gate_rows"])
        else:
            state["op"] = nn.GatedFFN(case["width"], case["hidden"], workers=case["workers"], max_rows=case["tokens"],
                                      dtype=dtype, activation=nn.ACTIVATIONS[case["activation"]], train=case["train"])
    torch.cuda.synchronize()
    return state


def run(state):
    case, t = state["case"], state["t"]
    if own:
        return {"clip": _own_clip, "norm": _own_norm, "ffn": _own_ffn}[case["op"]](state["op"], case, t)
    return {"clip": _plain_clip, "norm": _plain_norm, "ffn": _plain_ffn}[case["op"]](case, t)


# ---- as a user of the framework calls them -------------------------------------------------------------------------

def _own_clip(op, case, t):
    out, norm = op.clip(t["grad"], t["max_norm"], out=t["out"], scale=case["scale"])
    return dict(out=out, norm=norm)


def _own_norm(op, case, t):
    tensors = {k: t.get(k) for k in ("branch", "gate", "post", "pre", "post_bias", "pre_bias")}
    r, n = op.forward(t["residual"], **tensors)
    out = dict(residual=r, normed=n)
    if case["train"]:
        out.update(op.backward(t["d_residual"], t["d_normed"], t["residual"], **tensors))
    return out


def _own_ffn(op, case, t):
    if not case["train"]:
        return dict(y=op.forward(t["x"], t["w_gate"], t["w_up"], t["w_down"]))
    y, saved = op.forward(t["x"], t["w_gate"], t["w_up"], t["w_down"], save=True)
    dx, dg, du, dd = op.backward(t["dy"], t["x"], t["w_gate"], t["w_up"], t["w_down"], saved)
    return dict(y=y, dx=dx, dw_gate=dg, dw_up=du, dw_down=dd)


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ---------------------------------------

def _plain_clip(case, t):
    g = torch.where(t["real"], t["grad"].float(), 0.0)
    norm = (g * g).sum(1).sqrt() * case["scale"]
    keep = (t["max_norm"] / (norm + 1e-6)).clamp(max=1.0) * case["scale"]
    return dict(out=(g * keep[:, None]).to(t["out"].dtype), norm=norm)


def _plain_unit(case, x):
    """x normalised over its last axis, and what that divided by."""
    if case["kind"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    inv = 1.0 / ((x * x).mean(-1, keepdim=True) + EPS).sqrt()
    return x * inv, inv


def _plain_unit_grad(case, dunit, unit, inv):
    d = dunit - unit * (dunit * unit).mean(-1, keepdim=True)
    if case["kind"] == "layer":
        d = d - dunit.mean(-1, keepdim=True)
    return d * inv


def _plain_norm(case, t):
    dtype = t["residual"].dtype
    f = {k: v.float() for k, v in t.items()}
    layer, tokens, group = case["kind"] == "layer", case["tokens"], case["gate_rows"]
    after, gate = f["branch"], 1.0
    if case["post"]:
        unit_b, inv_b = _plain_unit(case, f["branch"])
        after = unit_b * f["post"][:, None]
        if layer:
            after = after + f["post_bias"][:, None]
    if group:
        which = torch.arange(tokens, device=after.device) // group
        gate = f["gate"][:, which]
    r = RESIDUAL * f["residual"] + BRANCH * gate * after
    unit_r, inv_r = _plain_unit(case, r)
    n = unit_r * f["pre"][:, None]
    if layer:
        n = n + f["pre_bias"][:, None]
    out = dict(residual=r, normed=n)
    if case["train"]:
        dn = f["d_normed"]
        out["d_pre"] = (dn * unit_r).sum(1)
        if layer:
            out["d_pre_bias"] = dn.sum(1)
        dr = f["d_residual"] + _plain_unit_grad(case, dn * f["pre"][:, None], unit_r, inv_r)
        out["d_residual"] = RESIDUAL * dr
        if group:
            dgate = BRANCH * dr * after
            out["d_gate"] = torch.zeros_like(f["gate"]).index_add_(1, which, dgate)
        dafter = BRANCH * gate * dr
        if case["post"]:
            out["d_post"] = (dafter * unit_b).sum(1)
            if layer:
                out["d_post_bias"] = dafter.sum(1)
            dafter = _plain_unit_grad(case, dafter * f["post"][:, None], unit_b, inv_b)
        out["d_branch"] = dafter
    return {k: v.to(dtype) for k, v in out.items()}


def _plain_act(kind, g):
    """The activation and its derivative."""
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if kind == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(g * 0.5 ** 0.5))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5
    if kind == "gelu_tanh":
        c = (2.0 / math.pi) ** 0.5
        th = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * c * (1.0 + 3 * 0.044715 * g * g)
    return g.clamp(min=0.0), (g > 0).float()


def _plain_ffn(case, t):
    dtype = t["x"].dtype
    x, wg, wu, wd = (t[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    g, u = x @ wg.mT, x @ wu.mT
    a, slope = _plain_act(case["activation"], g)
    h = a * u
    out = dict(y=h @ wd.mT)
    if case["train"]:
        dy = t["dy"].float()
        dh = dy @ wd
        dg, du = dh * u * slope, dh * a
        out.update(dx=dg @ wg + du @ wu, dw_gate=dg.mT @ x, dw_up=du.mT @ x, dw_down=dy.mT @ h)
    return {k: v.to(dtype) for k, v in out.items()}


# ---- the definitions in 64 bits; gradients come from differentiating them --------------------------------------------

def exact(case, seed):
    t = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    return {"clip": _exact_clip, "norm": _exact_norm, "ffn": _exact_ffn}[case["op"]](case, t)


def _exact_clip(case, t):
    out, norms = torch.zeros_like(t["out"]), []
    for g, o in zip(t["grad"], out):
        total = 0.0
        pieces = [slice(at, at + n) for at, n in zip(_places(case)[0], _numel(case))]
        for p in pieces:
            total += float(torch.dot(g[p], g[p]))
        norm = abs(case["scale"]) * math.sqrt(total)
        norms.append(norm)
        for p in pieces:
            o[p] = g[p] * (case["scale"] * min(1.0, t["max_norm"] / (norm + 1e-6)))
    return dict(out=out, norm=torch.tensor(norms, dtype=torch.float64))


def _exact_norm(case, t):
    names = [k for k in ("residual", "branch", "gate", "post", "pre", "post_bias", "pre_bias") if k in t]
    results = []
    for w in range(case["workers"]):
        v = {k: t[k][w].clone().requires_grad_(case["train"]) for k in names}

        def norm(z, name):
            if case["kind"] == "layer":
                return (z - z.mean(-1, keepdim=True)) / torch.sqrt(z.var(-1, unbiased=False, keepdim=True) + EPS) * v[name] + v[name + "_bias"]
            return z / torch.sqrt(z.pow(2).mean(-1, keepdim=True) + EPS) * v[name]

        z = norm(v["branch"], "post") if case["post"] else v["branch"]
        if "gate" in v:
            z = z * v["gate"].repeat_interleave(case["gate_rows"], 0)[:case["tokens"]]
        r = RESIDUAL * v["residual"] + BRANCH * z
        n = norm(r, "pre")
        out = dict(residual=r.detach(), normed=n.detach())
        if case["train"]:
            grads = torch.autograd.grad([r, n], [v[k] for k in names], [t["d_residual"][w], t["d_normed"][w]])
            out.update({"d_" + k: g for k, g in zip(names, grads)})
        results.append(out)
    return {k: torch.stack([o[k] for o in results]) for k in results[0]}


def _exact_ffn(case, t):
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu,
           "gelu_tanh": lambda g: torch.nn.functional.gelu(g, approximate="tanh")}[case["activation"]]
    names = ("x", "w_gate", "w_up", "w_down")
    results = []
    for w in range(case["workers"]):
        x, wg, wu, wd = (t[k][w].clone().requires_grad_(case["train"]) for k in names)
        y = (act(x @ wg.t()) * (x @ wu.t())) @ wd.t()
        out = dict(y=y.detach())
        if case["train"]:
            grads = torch.autograd.grad(y, (x, wg, wu, wd), t["dy"][w])
            out.update({"d" + k: g for k, g in zip(names, grads)})
        results.append(out)
    return {k: torch.stack([o[k] for o in results]) for k in results[0]}
