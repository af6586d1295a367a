"""Embeddings, routers, experts' order and orthogonal updates in 64 bits on the CPU, with bounds of what 32-bit kernels may be off.

Written from the formulas with plain loops.  Bounds as in nn_reference: a sum of n terms in any order is off by at most n * 2^-24 times the sum of their
magnitudes, a rounding to p bits by 2^-p of the value (and half the smallest subnormal), a library function by 8 units of 2^-24.
"""
import math

import torch

from nn_reference import FUNCTION, U32, rounding


def embed(ids, table, scale, dtype):
    """One worker's rows and their bound."""
    real = (ids >= 0) & (ids < table.shape[0])
    y = torch.where(real[:, None], scale * table[torch.where(real, ids, 0)], 0.0)
    return y, U32 * y.abs() + rounding(y, dtype)


def embed_backward(ids, dy, vocab, scale, dtype, old=None):
    """One worker's gradient of the table and its bound."""
    total, size = torch.zeros(vocab, dy.shape[1], dtype=torch.float64), torch.zeros(vocab, dy.shape[1], dtype=torch.float64)
    count = torch.zeros(vocab, 1, dtype=torch.float64)
    for t, v in enumerate(ids.tolist()):
        if 0 <= v < vocab:
            total[v] += dy[t]
            size[v] += dy[t].abs()
            count[v] += 1
    value = scale * total + (0.0 if old is None else old)
    error = (count + 1) * U32 * abs(scale) * size + (0.0 if old is None else 2 * U32 * (value.abs() + old.abs()))
    return value, error + rounding(value.abs() + error, dtype)


def choose(logits, top):
    """The chosen experts of every row, by a loop over the definition: the largest first, ties to the lowest number, a NaN first of all."""
    out = torch.full((*logits.shape[:-1], top), -1, dtype=torch.int32)
    for at, row in enumerate(logits.reshape(-1, logits.shape[-1]).tolist()):
        order = sorted((e for e, v in enumerate(row) if v != -math.inf), key=lambda e: (0 if row[e] != row[e] else 1, -row[e] if row[e] == row[e] else 0, e))
        for k, e in enumerate(order[:top]):
            out.view(-1, top)[at, k] = e
    return out


def route(logits, chosen, over_chosen, dw=None, dtype=None):
    """(weights, bound) and, from dw, (d_logits, bound); finite logits or minus infinity."""
    there = chosen >= 0
    at = chosen.long().clamp(min=0)
    counts = torch.zeros_like(logits).scatter_add_(-1, at, there.double()) > 0
    inside = torch.where(counts, logits, -math.inf) if over_chosen else logits
    most = inside.amax(-1, keepdim=True)
    most = torch.where(most > -math.inf, most, 0.0)
    e = torch.exp(inside - most)
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / torch.where(total > 0, total, 1.0), 0.0)
    # the exponent's difference rounds once, the function is a few units off, the sum of n terms n, the quotient once
    n = logits.shape[-1]
    far = torch.where(inside > -math.inf, (most - inside).abs(), 0.0)
    spread = torch.where(e > 0, far * e, 0.0).sum(-1, keepdim=True) / torch.where(total > 0, total, 1.0)
    rel = (far + spread + n + 2) * U32 + 2 * FUNCTION
    tiny = 2.0 ** -126   # below it the function may give 0
    w, ew = torch.where(there, p.gather(-1, at), 0.0), torch.where(there, (p * rel).gather(-1, at) + tiny, 0.0)
    if dw is None:
        return w, ew
    dw = torch.where(there, dw, 0.0)
    inner = (w * dw).sum(-1, keepdim=True)
    e_inner = ((ew + n * U32 * w) * dw.abs()).sum(-1, keepdim=True)
    sent = torch.zeros_like(logits).scatter_add_(-1, at, dw)
    d = p * (sent - inner)
    ed = (p * rel + tiny) * ((sent - inner).abs() + e_inner) + p * (e_inner + 2 * U32 * (sent.abs() + inner.abs())) + 2 * U32 * d.abs()
    return w, ew, d, ed + rounding(d.abs() + ed, dtype)


def plan(chosen, experts, capacity):
    """One worker's (slot, source, counts) by a loop over its entries."""
    flat = chosen.reshape(-1).tolist()
    counts = [0] * experts
    for e in flat:
        if 0 <= e < experts:
            counts[e] += 1
    first = [e * capacity if capacity else sum(counts[:e]) for e in range(experts)]
    slot, source = [-1] * len(flat), [-1] * (experts * capacity if capacity else len(flat))
    seen = [0] * experts
    for i, e in enumerate(flat):
        if 0 <= e < experts:
            if not capacity or seen[e] < capacity:
                slot[i] = first[e] + seen[e]
                source[slot[i]] = i
            seen[e] += 1
    whole = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return whole(slot).view(chosen.shape), whole(source), whole(counts)


def dispatch(x, source, top):
    real = source >= 0
    if not len(x):
        return x.new_zeros(len(source), x.shape[1])
    return torch.where(real[:, None], x[source.long().clamp(min=0) // top], torch.zeros((), dtype=x.dtype))


def combine(rows, weights, slot, dtype):
    """(y, bound) of one worker; weights None: all 1."""
    T, K = slot.shape
    if not T:
        none = torch.zeros(0, rows.shape[1], dtype=torch.float64)
        return none, none
    real = (slot >= 0)[..., None]
    r = torch.where(real, rows[slot.long().clamp(min=0)], 0.0)
    w = torch.ones(T, K, 1, dtype=torch.float64) if weights is None else weights[..., None]
    terms = torch.where(real, w * r, 0.0)
    y, size = terms.sum(1), terms.abs().sum(1)
    e = (K + 1) * U32 * size
    return y, e + rounding(y.abs() + e, dtype)


def combine_backward(dy, rows, weights, slot, source, top, dtype):
    """((d_rows, bound), (d_weights, bound)) of one worker."""
    if not len(dy):
        none = torch.zeros(len(source), dy.shape[1], dtype=torch.float64)
        return (none, none), (weights, weights)
    real = source >= 0
    entry = source.long().clamp(min=0)
    d = torch.where(real[:, None], weights.reshape(-1)[entry][:, None] * dy[entry // top], 0.0)
    terms = torch.where((slot >= 0)[..., None], dy[:, None] * rows[slot.long().clamp(min=0)], 0.0)
    return (d, U32 * d.abs() + rounding(d, dtype)), (terms.sum(-1), (dy.shape[-1] + 1) * U32 * terms.abs().sum(-1))


# ---- orthogonal updates --------------------------------------------------------------------------------------------------------

HALF = 2.0 ** -11            # a rounding to float16
KEPT = 2.0 ** -22            # what two parts of it leave
POLYNOMIAL = (3.4445, -4.7750, 2.0315)


def momentum(grad, old, mu, nesterov):
    """(m', u)"""
    m = mu * old + grad
    return m, grad + mu * m if nesterov else m


def _through(f, s):
    """The largest divided difference of an odd function f over the singular values s and their negatives, zero included: the largest factor by which
    f of a matrix with these singular values changes more than the matrix does, to first order, in the Frobenius norm."""
    v = torch.cat([s, -s, torch.zeros(1, dtype=s.dtype)])
    a, b = v[:, None], v[None, :]
    near = (a - b).abs() < 1e-4
    step = 1e-5
    slope = (f(v + step) - f(v - step)) / (2 * step)
    return float(torch.where(near, slope.abs()[:, None].expand_as(near), (f(a) - f(b)).abs() / torch.where(near, 1.0, (a - b).abs())).max())


def orthogonal(u, dtype, *, steps=5, polynomial=POLYNOMIAL, eps=1e-7, scale=1.0):
    """(update, bound of the Frobenius norm of what it may be off) of one matrix.

    A step's own error is at most (first order, Frobenius norms, |.|_2 the largest singular value, n and k the sides, o the rounding of an operand: float16's, or
    of two parts of it 2^-22 twice, as the product of the second parts is left out):
        dS = 2 o |X|_2 |X| + k 2^-24 |X|^2 + o |S|
        dP = |b| dS + |c| (2 |S|_2 dS + 2 o |S|_2 |S| + n 2^-24 |S|^2) + o |P|
        dX = |a| (2^-22 + 2^-24) |X| + |X|_2 dP + 2 o |P|_2 |X| + n 2^-24 |P| |X| + 2^-22 |X'|
    and what a step has left grows through the steps behind it by at most _through of them.
    """
    a, b, c = polynomial
    o = 2 * KEPT if dtype == torch.float32 else HALF
    p = lambda s: s * (a + s * s * (b + s * s * c))  # noqa: E731
    x = u / (u.norm() + eps)
    n, k = min(x.shape), max(x.shape)
    s = torch.linalg.svdvals(x)
    errors, values = [4 * U32 + KEPT], [s]   # norm, quotient, product; kept in two parts
    for _ in range(steps):
        S = x @ x.T if x.shape[0] <= x.shape[1] else x.T @ x
        P = b * S + c * S @ S
        F, top = float(x.norm()), float(s.max())
        fS, fP, topS, topP = float(S.norm()), float(P.norm()), top * top, float((b * s ** 2 + c * s ** 4).abs().max())
        dS = 2 * o * top * F + k * U32 * F * F + o * fS
        dP = abs(b) * dS + abs(c) * (2 * topS * dS + 2 * o * topS * fS + n * U32 * fS * fS) + o * fP
        x = a * x + (P @ x if x.shape[0] <= x.shape[1] else x @ P)
        s = p(s).abs()
        errors.append(abs(a) * (KEPT + U32) * F + top * dP + 2 * o * topP * F + n * U32 * fP * F + KEPT * float(x.norm()))
        values.append(s)
    total = 0.0
    for i, e in enumerate(errors):
        def rest(v, i=i):
            for _ in range(steps - i):
                v = p(v)
            return v
        total += e * _through(rest, values[i])
    out = scale * x
    return out, abs(scale) * 1.05 * total + float(rounding(out, torch.float32).norm() if dtype == torch.float32 else 0.0)
