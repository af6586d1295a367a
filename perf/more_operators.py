"""What a user of this framework has its operators for experts, tokens and orthogonal updates do, as cases that can be timed.

Four operators belong together: a ring worker's tokens become rows of its residual stream (`nn.Embedding`), a router gives each
token its experts and their weights (`nn.Router`), the tokens are sorted by expert, ahead of the experts' feed-forward
blocks, and brought back behind them (`nn.ExpertSort`), and the gradients of the matrices become orthogonal updates ahead of the ring's
step (`nn.Orthogonal`). All workers of a ring go in one call: tensors have the worker as their first axis.

For each worker:

    embed    y[t] = s * table[token[t]], 0 for tokens outside the table;  d_table[v] = s * sum of dy[t] where token[t] = v
    route    the K experts of the largest logits, the largest first, ties to the lowest; weights softmax(logits)[chosen], or
             the softmax over the chosen; experts at -inf are never chosen (-1, weight 0)
    experts  (t, k) sorted by expert: rows[slot] = x[t], y[t] = sum_k w[t, k] * done[slot[t, k]], and both gradients; slots are
             packed (capacity 0), or each expert has `capacity` of them and what exceeds it is left out
    update   m' = mu m + g, u = g + mu m', X = u / (|u| + eps), five times X <- a X + (b A + c A A) X with A = X X^T; s X
"""
import math

import numpy as np
import torch

own = False

_TYPE = dict(f32=torch.float32, f16=torch.float16, bf16=torch.bfloat16)
_SIZE = dict(f32=4, f16=2, bf16=2)
#: Elements of the largest listed table, sorted rows and logits; operations of the largest update.
MOST_TABLE = 50257 * 2048
MOST_SORTED = 16384 * 8 * 2048
MOST_LOGITS = 32768 * 128

#: The update's momentum, constants of its polynomial, steps, and what is added to the norm.
MOMENTUM, POLYNOMIAL, STEPS, EPS = 0.95, (3.4445, -4.7750, 2.0315), 5, 1e-7
#: What embeddings are scaled by.
EMBED = 0.75


def _embed(name, workers, tokens, vocab, width, dtype, train):
    return dict(name=name, op="embed", workers=workers, tokens=tokens, vocab=vocab, width=width, dtype=dtype, train=train)


def _route(name, workers, tokens, experts, top, dtype, over_chosen, masked, train):
    return dict(name=name, op="route", workers=workers, tokens=tokens, experts=experts, top=top, dtype=dtype, over_chosen=over_chosen,
                masked=masked, train=train)


def _experts(name, workers, tokens, experts, top, capacity, width, dtype, masked, train):
    return dict(name=name, op="experts", workers=workers, tokens=tokens, experts=experts, top=top, capacity=capacity, width=width,
                dtype=dtype, masked=masked, train=train)


def _update(name, matrices, rows, cols, dtype):
    return dict(name=name, op="update", matrices=matrices, rows=rows, cols=cols, dtype=dtype)


def listed():
    return [
        # one new token of one model
        _embed("embed_token", 1, 1, 32000, 2048, "bf16", False),
        # eight workers' short batches in 32 bits, as the ring holds its parameters; odd in every size
        _embed("embed_ring_f32", 8, 333, 1003, 785, "f32", True),
        # a long training batch: half of its tokens are of 224 words
        _embed("embed_train", 1, 16384, 50257, 2048, "bf16", True),
        # a prompt over few experts, an odd number of them, some switched off
        _route("route_prompt_f16", 1, 4097, 60, 4, "f16", False, 0.1, False),
        # a long training batch over many
        _route("route_train", 1, 32768, 128, 8, "bf16", True, 0.0, True),
        # one new token: its eight rows, and back
        _experts("experts_token", 1, 1, 64, 8, 0, 2048, "bf16", 0.0, False),
        # eight workers' batches in 32 bits, with room for a quarter more than an even share, padded tokens
        _experts("experts_ring_f32", 8, 250, 8, 2, 79, 785, "f32", 0.1, True),
        # a long training batch: every token at eight experts, none left out
        _experts("experts_train", 1, 16384, 64, 8, 0, 2048, "bf16", 0.0, True),
        # the smallest ring that is trained, a perceptron on four workers: its first matrix, in 32 bits
        _update("update_mlp_p4_f32", 4, 128, 784, "f32"),
        # eight small workers' blocks, an odd hidden width
        _update("update_ring_f16", 8, 1365, 512, "f16"),
        # one matrix of a feed-forward block in 32 bits
        _update("update_block_f32", 1, 2048, 5632, "f32"),
        # a wide block's matrix
        _update("update_wide", 1, 4096, 11264, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _width(rng, lo, hi):
    """Widths are mostly whole cache lines; one in three is any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 1 / 3 else max(lo, n // 64 * 64)


def draw(rng):
    """One of the operators over the range of its listed cases: rings of 1 to 16 workers, one token to long batches, small
    matrices to wide ones, any number between."""
    most_flops = max(work(c)["flops"] for c in listed())
    while True:
        op = rng.choice(("embed", "route", "experts", "update"))
        workers, dtype = rng.choice((1, 1, _log_int(rng, 2, 16))), rng.choice(("bf16", "bf16", "f16", "f32"))
        if op == "embed":
            case = _embed("", workers, _log_int(rng, 1, 16384), _log_int(rng, 64, 131072), _width(rng, 64, 4096), dtype, rng.random() < 0.6)
            fits = workers * max(case["vocab"], case["tokens"]) * case["width"] * _SIZE[dtype] <= 2 * MOST_TABLE
        elif op == "route":
            experts = _log_int(rng, 2, 256)
            case = _route("", workers, _log_int(rng, 1, 32768), experts, rng.randint(1, min(8, experts)), dtype, rng.random() < 0.5,
                          rng.choice((0.0, 0.0, 0.2)), rng.random() < 0.5)
            fits = workers * case["tokens"] * experts <= MOST_LOGITS
        elif op == "experts":
            experts, tokens = _log_int(rng, 2, 256), _log_int(rng, 1, 16384)
            top = rng.randint(1, min(8, experts))
            capacity = 0 if rng.random() < 0.5 else math.ceil(rng.uniform(1.0, 1.5) * tokens * top / experts)
            case = _experts("", workers, tokens, experts, top, capacity, _width(rng, 64, 4096), dtype, rng.choice((0.0, 0.0, 0.2)),
                            rng.random() < 0.6)
            fits = workers * _slots(case) * case["width"] * _SIZE[dtype] <= 2 * MOST_SORTED
        else:
            case = _update("", workers, _width(rng, 16, 8192), _width(rng, 16, 8192), dtype)
            # 32-bit products go at a sixteenth of the rate
            fits = work(case)["flops"] * (16 if dtype == "f32" else 1) <= most_flops
        if fits:
            del case["name"]
            return case


def _slots(case):
    return case["experts"] * case["capacity"] if case["capacity"] else case["tokens"] * case["top"]


def _distinct(case):
    """How many rows of a table a worker's tokens are expected to name: they are spread evenly over the logarithm of their number."""
    v = np.arange(case["vocab"], dtype=np.float64)
    p = np.log1p(1.0 / (v + 1.0)) / math.log(case["vocab"] + 1.0)
    return float(np.sum(-np.expm1(case["tokens"] * np.log1p(-np.minimum(p, 1 - 1e-16)))))


def work(case):
    e = _SIZE[case["dtype"]]
    if case["op"] == "update":
        n, m, count = min(case["rows"], case["cols"]), max(case["rows"], case["cols"]), case["matrices"]
        # A and A A are symmetric: half of each
        return {"bytes": float(count * n * m * (2 * e + 8)), "flops": float(count * STEPS * (n * n * m + n * n * n + 2 * n * n * m))}
    rows = case["workers"] * case["tokens"]
    if case["op"] == "embed":
        d = case["width"]
        values, flops = rows * d + case["workers"] * _distinct(case) * d, rows * d
        if case["train"]:
            values, flops = values + rows * d + case["workers"] * case["vocab"] * d, flops + 2 * rows * d
        return {"bytes": float(e * values + 8 * rows), "flops": float(flops)}
    if case["op"] == "route":
        logits, top = rows * case["experts"], rows * case["top"]
        if not case["train"]:
            return {"bytes": float(e * logits + 8 * top), "flops": 4.0 * logits}
        return {"bytes": float(2 * e * logits + 12 * top), "flops": 8.0 * logits}
    d, top, slots = case["width"], rows * case["top"], case["workers"] * _slots(case)
    moved = min(top, slots)
    values, words = 2 * rows * d + (slots + moved) * d, 2 * top + 2 * top + slots
    if case["train"]:
        values, words = values + 2 * rows * d + (slots + moved) * d, words + top
    return {"bytes": float(e * values + 4 * words), "flops": float((5 if case["train"] else 2) * moved * d)}


def _inputs(case, seed):
    """Tensors of the case on the GPU, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = _TYPE[case["dtype"]]

    def normal(*shape, size=1.0, kind=dtype):
        return torch.empty(shape, dtype=kind, device="cuda").normal_(generator=gen).mul_(size)

    def share(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    if case["op"] == "update":
        # gradients of matrices: a few directions carry most of them, the others are there all the same
        w, r, c = case["matrices"], case["rows"], case["cols"]
        rank = max(1, min(r, c) // 16)
        left = normal(w, r, rank, kind=torch.float32) * torch.exp(torch.linspace(0, -3, rank, device="cuda"))

        def gradient():
            return (torch.bmm(left, normal(w, rank, c, kind=torch.float32)) / rank ** 0.5 + normal(w, r, c, size=0.1, kind=torch.float32)) * 1e-3

        return dict(grad=gradient().to(dtype), momentum=gradient() * 8)
    workers, tokens = case["workers"], case["tokens"]
    if case["op"] == "embed":
        ids = torch.floor(torch.exp(share(workers, tokens) * math.log(case["vocab"] + 1.0)) - 1.0).long().clamp_(0, case["vocab"] - 1)
        if tokens > 8:
            ids[:, -(tokens // 8):][share(workers, tokens // 8) < 0.5] = -1  # the padding behind a batch's shorter sequences
        t = dict(ids=ids, table=normal(workers, case["vocab"], case["width"], size=0.02))
        if case["train"]:
            t["dy"] = normal(workers, tokens, case["width"])
        return t
    experts, top = case["experts"], case["top"]
    if case["op"] == "route":
        logits = normal(workers, tokens, experts, size=2.0)
        if case["masked"]:
            logits[share(workers, tokens, experts) < case["masked"]] = -math.inf
            logits[share(workers, tokens) < 0.05] = -math.inf  # tokens that no expert is to see
        t = dict(logits=logits)
        if case["train"]:
            t["d_weights"] = normal(workers, tokens, top, kind=torch.float32)
        return t
    # some experts are asked for more often than others
    liking = torch.randn(workers, 1, experts, generator=gen, device="cuda") * 0.5
    scores = liking + torch.randn(workers, tokens, experts, generator=gen, device="cuda")
    best, chosen = scores.topk(top, dim=-1)
    chosen = chosen.int()
    chosen[share(workers, tokens) < case["masked"]] = -1
    d = case["width"]
    t = dict(x=normal(workers, tokens, d), chosen=chosen, weights=torch.softmax(best, -1), done=normal(workers, _slots(case), d))
    if case["train"]:
        t.update(dy=normal(workers, tokens, d), d_rows=normal(workers, _slots(case), d))
    return t


def prepare(case, seed):
    """The tensors that a pass reads, and the operator's handle where it has one."""
    state = dict(case=case, t=_inputs(case, seed))
    if own:
        from paper_2103_07454_amd import nn
        dtype = _TYPE[case["dtype"]]
        if case["op"] == "embed":
            state["op"] = nn.Embedding(case["vocab"], case["width"], workers=case["workers"], max_tokens=case["tokens"], dtype=dtype,
                                       scale=EMBED, train=case["train"])
        elif case["op"] == "route":
            state["op"] = nn.Router(case["experts"], case["top"], workers=case["workers"], max_tokens=case["tokens"], dtype=dtype,
                                    over_chosen=case["over_chosen"])
        elif case["op"] == "experts":
            state["op"] = nn.ExpertSort(case["experts"], case["top"], case["width"], workers=case["workers"], max_tokens=case["tokens"],
                                        capacity=case["capacity"], dtype=dtype)
        else:
            state["op"] = nn.Orthogonal(case["rows"], case["cols"], matrices=case["matrices"], dtype=dtype, momentum=MOMENTUM,
                                        nesterov=True, polynomial=POLYNOMIAL, steps=STEPS, eps=EPS, scale=_update_scale(case))
    if case["op"] == "update":
        state["momentum"] = torch.empty_like(state["t"]["momentum"])
    torch.cuda.synchronize()
    return state


def _update_scale(case):
    """Updates of tall matrices are longer, so that outputs change alike."""
    return max(1.0, case["rows"] / case["cols"]) ** 0.5


def run(state):
    case, t = state["case"], state["t"]
    if own:
        return {"embed": _own_embed, "route": _own_route, "experts": _own_experts, "update": _own_update}[case["op"]](state, case, t)
    return {"embed": _plain_embed, "route": _plain_route, "experts": _plain_experts, "update": _plain_update}[case["op"]](state, case, t)


# ---- as a user of the framework calls them -------------------------------------------------------------------------

def _own_embed(state, case, t):
    op = state["op"]
    out = dict(y=op.forward(t["ids"], t["table"]))
    if case["train"]:
        out["d_table"] = op.backward(t["dy"], t["ids"])
    return out


def _own_route(state, case, t):
    op = state["op"]
    chosen, weights = op.forward(t["logits"])
    out = dict(chosen=chosen, weights=weights)
    if case["train"]:
        out["d_logits"] = op.backward(t["d_weights"], t["logits"], chosen)
    return out


def _own_experts(state, case, t):
    op = state["op"]
    rows, plan = op.dispatch(t["x"], t["chosen"])
    out = dict(rows=rows, slot=plan.slot, source=plan.source, counts=plan.counts, y=op.combine(t["done"], t["weights"], plan))
    if case["train"]:
        out["d_done"], out["d_weights"] = op.combine_backward(t["dy"], t["done"], t["weights"], plan)
        out["dx"] = op.dispatch_backward(t["d_rows"], plan)
    return out


def _own_update(state, case, t):
    out = state["op"].update(t["grad"], momentum=t["momentum"], momentum_out=state["momentum"])
    return dict(update=out, momentum=state["momentum"])


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ---------------------------------------

def _plain_embed(state, case, t):
    workers, vocab, width = t["table"].shape
    ids = t["ids"]
    real = (ids >= 0) & (ids < vocab)
    at = (torch.where(real, ids, 0) + torch.arange(workers, device=ids.device)[:, None] * vocab).flatten()
    y = t["table"].view(-1, width)[at].float() * EMBED * real.flatten()[:, None]
    out = dict(y=y.view(workers, -1, width).to(t["table"].dtype))
    if case["train"]:
        d = t["dy"].float().view(-1, width) * real.flatten()[:, None]
        table = torch.zeros(workers * vocab, width, device=d.device).index_add_(0, at, d)
        out["d_table"] = (table * EMBED).view(workers, vocab, width).to(t["table"].dtype)
    return out


def _plain_route(state, case, t):
    logits = t["logits"].float()
    ordered, at = torch.sort(logits, dim=-1, descending=True, stable=True)
    best, chosen = ordered[..., :case["top"]], at[..., :case["top"]]
    there = best > -math.inf
    top = torch.where(there[..., :1], ordered[..., :1], 0.0)  # nothing is left of a row without experts
    e = torch.exp(best - top)
    total = (e if case["over_chosen"] else torch.exp(logits - top)).sum(-1, keepdim=True)
    w = torch.where(there, e / total, 0.0)
    out = dict(chosen=torch.where(there, chosen, -1).int(), weights=w)
    if case["train"]:
        dw = torch.where(there, t["d_weights"], 0.0)
        inner = (w * dw).sum(-1, keepdim=True)
        if case["over_chosen"]:
            d = torch.zeros_like(logits).scatter_(-1, chosen, w * (dw - inner))
        else:
            p = torch.where(there[..., :1], torch.exp(logits - top) / total, 0.0)
            d = p * (torch.zeros_like(logits).scatter_(-1, chosen, dw) - inner)
        out["d_logits"] = d.to(t["logits"].dtype)
    return out


def _plain_experts(state, case, t):
    workers, tokens, width = t["x"].shape
    experts, top, capacity, slots, dev = case["experts"], case["top"], case["capacity"], _slots(case), t["x"].device
    key = t["chosen"].reshape(workers, -1).long()
    key = torch.where(key < 0, experts, key)
    ordered, order = torch.sort(key, dim=1, stable=True)
    counts = torch.zeros(workers, experts + 1, dtype=torch.long, device=dev).scatter_add_(1, key, torch.ones_like(key))
    start = counts.cumsum(1) - counts
    rank = torch.arange(tokens * top, device=dev) - start.gather(1, ordered)
    fits = (ordered < experts) & ((rank < capacity) if capacity else True)
    place = ordered * capacity + rank if capacity else start.gather(1, ordered) + rank
    slot = torch.full_like(key, -1).scatter_(1, order, torch.where(fits, place, -1))
    source = torch.full((workers, slots + 1), -1, dtype=torch.long, device=dev)
    source = source.scatter_(1, torch.where(fits, place, slots), torch.where(fits, order, -1))[:, :slots]
    base = torch.arange(workers, device=dev)[:, None]
    filled = (source >= 0).flatten()
    token = (source.clamp(min=0) // top + base * tokens).flatten()
    rows = t["x"].view(-1, width)[token] * filled[:, None]
    sent = (slot >= 0).flatten()
    where = (slot.clamp(min=0) + base * slots).flatten()
    w = t["weights"].reshape(-1)
    done = t["done"].view(-1, width)[where].float() * sent[:, None]
    y = (done * w[:, None]).view(workers, tokens, top, width).sum(2)
    out = dict(rows=rows.view(workers, slots, width), slot=slot.view(workers, tokens, top).int(), source=source.int(),
               counts=counts[:, :experts].int(), y=y.to(t["x"].dtype))
    if case["train"]:
        dy = t["dy"].float()
        weight = t["weights"].view(workers, -1).gather(1, source.clamp(min=0)).flatten() * filled
        out["d_done"] = (dy.view(-1, width)[token] * weight[:, None]).view(workers, slots, width).to(t["x"].dtype)
        out["d_weights"] = (done.view(workers, tokens, top, width) * dy[:, :, None]).sum(-1)
        back = t["d_rows"].view(-1, width)[where].float() * sent[:, None]
        out["dx"] = back.view(workers, tokens, top, width).sum(2).to(t["x"].dtype)
    return out


def _plain_update(state, case, t):
    a, b, c = POLYNOMIAL
    g = t["grad"].float()
    m = MOMENTUM * t["momentum"] + g
    state["momentum"].copy_(m)
    x = g + MOMENTUM * m
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + EPS)
    if case["rows"] > case["cols"]:
        x = x.mT.contiguous()
    for _ in range(STEPS):
        s = torch.bmm(x, x.mT)
        x = a * x + torch.bmm(b * s + c * torch.bmm(s, s), x)
    if case["rows"] > case["cols"]:
        x = x.mT
    return dict(update=(x * _update_scale(case)).to(t["grad"].dtype).contiguous(), momentum=state["momentum"])


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    t = {k: v.double() if v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    return {"embed": _exact_embed, "route": _exact_route, "experts": _exact_experts, "update": _exact_update}[case["op"]](case, t)


def _exact_embed(case, t):
    out = dict(y=torch.zeros(case["workers"], case["tokens"], case["width"], dtype=torch.float64, device="cuda"))
    if case["train"]:
        out["d_table"] = torch.zeros_like(t["table"])
    for w, ids in enumerate(t["ids"]):
        here = ((ids >= 0) & (ids < case["vocab"])).nonzero()[:, 0]
        out["y"][w, here] = EMBED * t["table"][w].index_select(0, ids[here])
        if case["train"]:
            here = here[torch.argsort(ids[here], stable=True)]
            values, lengths = torch.unique_consecutive(ids[here], return_counts=True)
            out["d_table"][w, values] = EMBED * torch.segment_reduce(t["dy"][w][here], "sum", lengths=lengths, axis=0, unsafe=True)
    return out


def _exact_route(case, t):
    logits = t["logits"].clone().requires_grad_(case["train"])
    _, at = torch.sort(t["logits"], dim=-1, descending=True, stable=True)
    chosen = at[..., :case["top"]]
    best = logits.gather(-1, chosen)
    there = best.detach() > -math.inf
    some = there.any(-1, keepdim=True)
    over = best if case["over_chosen"] else logits
    log_w = best - torch.logsumexp(torch.where(some, over, 0.0), -1, keepdim=True)
    w = torch.where(there, torch.where(there, log_w, 0.0).exp(), 0.0)
    out = dict(chosen=torch.where(there, chosen, -1).int(), weights=w.detach())
    if case["train"]:
        out["d_logits"] = torch.autograd.grad(w, logits, t["d_weights"])[0]
    return out


def _exact_experts(case, t):
    workers, tokens, width = t["x"].shape
    experts, top, slots = case["experts"], case["top"], _slots(case)
    zeros = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")  # noqa: E731
    whole = lambda *s: torch.full(s, -1, dtype=torch.int32, device="cuda")  # noqa: E731
    out = dict(rows=zeros(workers, slots, width), slot=whole(workers, tokens * top), source=whole(workers, slots),
               counts=whole(workers, experts), y=zeros(workers, tokens, width))
    if case["train"]:
        out.update(d_done=zeros(workers, slots, width), d_weights=zeros(workers, tokens * top), dx=zeros(workers, tokens, width))
    for w in range(workers):
        flat, weight = t["chosen"][w].flatten(), t["weights"][w].flatten()
        first = 0
        for e in range(experts):
            mine = (flat == e).nonzero()[:, 0]
            out["counts"][w, e] = mine.numel()
            if case["capacity"]:
                mine, first = mine[:case["capacity"]], e * case["capacity"]
            to = slice(first, first + mine.numel())
            first += mine.numel()
            token = mine // top
            out["slot"][w, mine] = torch.arange(to.start, to.stop, dtype=torch.int32, device="cuda")
            out["source"][w, to] = mine.int()
            out["rows"][w, to] = t["x"][w, token]
            # a token names an expert once, so no two of these rows meet
            out["y"][w, token] += weight[mine, None] * t["done"][w, to]
            if case["train"]:
                out["d_done"][w, to] = weight[mine, None] * t["dy"][w, token]
                out["d_weights"][w, mine] = (t["dy"][w, token] * t["done"][w, to]).sum(-1)
                out["dx"][w, token] += t["d_rows"][w, to]
    for k in ("slot", "d_weights"):
        if k in out:
            out[k] = out[k].view(workers, tokens, top)
    return out


def _exact_update(case, t):
    a, b, c = POLYNOMIAL
    results = []
    for g, old in zip(t["grad"], t["momentum"]):
        m = old * MOMENTUM + g
        x = m * MOMENTUM + g
        x = x / (torch.linalg.matrix_norm(x) + EPS)
        one = torch.eye(min(x.shape), dtype=x.dtype, device=x.device)
        for _ in range(STEPS):
            if x.shape[0] <= x.shape[1]:
                s = x @ x.T
                x = (a * one + s @ (b * one + c * s)) @ x
            else:
                s = x.T @ x
                x = x @ (a * one + s @ (b * one + c * s))
        results.append((x * max(1.0, case["rows"] / case["cols"]) ** 0.5, m))
    return dict(update=torch.stack([x for x, _ in results]), momentum=torch.stack([m for _, m in results]))
