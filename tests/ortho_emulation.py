"""What orthogonal updates come to in the arithmetic that their kernels are to have: float16 parts where those are kept or multiplied, 64 bits for all sums.

A kernel's sums are in 32 bits, in an order of its own.  What that may do to a result is found by emulating twice, the second time with every sum off by a
random amount: of K terms added one after the other, with partial sums that grow evenly to the value v and wander by r, r^2 the sum of the terms' squares, each
addition is off by at most 2^-24 of the partial sum, so that all are off by a standard deviation of at most 2^-24 sqrt(K) sqrt(v^2 + r^2).  Values next to the border between two
float16 (or two of the result's type) come to lie on the other side of it in both ways alike.  `tolerance` is four times the distance of the two results.

A mistake can be planted (`mistake`), which shows what a comparison within the tolerance would find.
"""
import math

import torch

from nn_reference import U32, UNIT

POLYNOMIAL = (3.4445, -4.7750, 2.0315)


def _single(v):
    return float(torch.tensor(v, dtype=torch.float32))


def _to(t, dtype):
    return t if dtype is None else t.to(torch.float32).to(dtype).to(t.dtype)


def _parts(t):
    """The nearest float16, and the nearest of what that leaves."""
    t = _to(t, torch.float32)
    hi = _to(t, torch.float16)
    return hi, _to(t - hi, torch.float16)


def _power(most):
    return 2.0 ** (15 - math.frexp(max(most, 1e-3))[1])


def _powers(polynomial, steps):
    """The powers of two that X, S and P are kept times."""
    a, b, c = polynomial
    s = lambda end: torch.linspace(0.0, end, 20001, dtype=torch.float64)  # noqa: E731
    bound = 1.01
    for _ in range(steps):
        v = s(bound)
        bound = max(bound, 1.01 * float((v * (a + v * v * (b + v * v * c))).abs().max()))
    v = s(bound * bound)
    return _power(bound), _power(bound * bound), _power(1.01 * float((b * v + c * v * v).abs().max()))


def emulate(u, both, out_dtype, *, steps=5, polynomial=POLYNOMIAL, eps=1e-7, scale=1.0, noise=None, mistake=None):
    """The update of one matrix u of 32-bit values, in 64 bits.  both: products of both parts of their operands.  noise: a generator for sums' errors."""
    a, b, c = (_single(v) for v in polynomial)
    tall = u.shape[0] > u.shape[1]
    u = (u.T if tall else u).double()
    kx, ks, kp = _powers((a, b, c), steps)
    f = _single(kx / (float(u.square().sum().sqrt()) + _single(eps)))
    X = _parts(u * f)

    def product(A, B, K, what):
        if mistake == "a share of k" and what == "square":     # the last eighth of what S S adds up
            keep = K - K // 8
            A, B = [t[:, :keep] for t in A], [t[:keep] for t in B]
        v = A[0] @ B[0]
        if both and mistake != f"one part, {what}":
            v = v + A[0] @ B[1] + A[1] @ B[0]
        if mistake == "a tile" and what == "square":           # a corner of S S
            v[-(len(v) // 8 or 1):, -(len(v) // 8 or 1):] = 0
        if mistake == f"without {what}":
            v = torch.zeros_like(v)
        if noise is not None:
            r = A[0].square() @ B[0].square()
            v = v + U32 * math.sqrt(K) * (v.square() + r).sqrt() * torch.randn(v.shape, generator=noise, dtype=v.dtype, device=v.device)
        return v

    def kept(v):
        hi, lo = _parts(v)
        return hi, lo if both else torch.zeros_like(lo)

    n, k = u.shape
    for i in range(steps):
        S = kept(product(X, [t.T for t in X], k, "gram") * _single(ks / (kx * kx)))
        P = kept(product(S, S, n, "square") * _single(c * kp / (ks * ks)) + (S[0] + S[1]) * _single(b * kp / ks))
        new = product(P, X, n, "apply") / kp
        if mistake == "X in one part":
            X = X[0], torch.zeros_like(X[1])
        new = new + (X[0] + X[1]) * a
        if i + 1 < steps:
            X = _parts(new)
    out = _to(new * (_single(scale) / kx), out_dtype)
    return out.T if tall else out


def tolerance(want, u, both, out_dtype, *, seed=0, **options):
    """How far (Frobenius norm) a result may be from `want`, what `emulate` makes of the same arguments."""
    noise = torch.Generator(device=u.device).manual_seed(seed)
    off = float((emulate(u, both, out_dtype, noise=noise, **options) - want).norm())
    # Results' own borders: few matrices' elements may have none near one in this run of the noise and two in a kernel.
    return 4 * off + 4 * UNIT[out_dtype] * float(want.abs().max())


def gradient(gen, *shape):
    """A few strong directions, singular values of the normed matrix of about a half, and weaker ones of every kind: both S S and what grows from the smallest values show in the result."""
    w, r, c = shape
    k = min(3, r, c)
    make = lambda *s: torch.randn(*s, generator=gen, device=gen.device)  # noqa: E731
    strong = torch.bmm(make(w, r, k), make(w, k, c)) / k ** 0.5
    return 1e-3 * (strong + 0.5 * make(w, r, c))
