"""Ring workers that train a small language model with experts: the operators of ``nn`` from tokens to the ring's step.

Every worker has its own copy of the parameters in the ring's arena and its own tokens.  A step runs, for all workers at once,

    forward     Embedding; for each block BlockNorm, Router, ExpertSort.dispatch, a GatedFFN for each expert, ExpertSort.combine; the last
                BlockNorm, and logits over the vocabulary by the embedding's own table
    backward    the same back, every parameter's gradient written where the ring looks for it
    clipping    GradClip: each worker's gradient to at most ``max_norm``, into the 32-bit arena
    updates     Orthogonal: the experts' matrices' part of that arena becomes orthogonal updates (with ``orthogonal``)
    the ring    Ring.step: triggers, sends, averaging with the neighbours and SGD

Each expert's matrices are tensors of their own, so that the ring's events are too: an expert that few tokens reach seldom sends.
The plain products, of the router's and the vocabulary's logits, and the loss are torch's, in 32 bits.

Tokens outside the vocabulary, as -1, are padding: rows of zeros, no experts, no loss; targets outside it have none either.  Types, the loss scale of float16 and streams are as in
``ffn_ring``.

    python -m paper_2103_07454_amd.mixture_ring --workers 4 --width 256 --hidden 512 --experts 8 --tokens 256 --dtype bf16
"""
from __future__ import annotations

import argparse
import math

import numpy as np
import torch

from . import evg, nn
from .ffn_ring import FFNRing


class MixtureRing(FFNRing):
    def __init__(self, workers=4, *, vocab=256, width=64, hidden=96, experts=4, top=2, capacity_factor=1.5, blocks=2, tokens=32, dtype=torch.float32,
                 activation="silu", lr=0.05, momentum=0.0, max_norm=1.0, orthogonal=True, orthogonal_scale=0.2, seed=0, loss_scale=None, device="cuda:0",
                 stream=None, **ring_options):
        if not capacity_factor > 0:
            raise ValueError("capacity_factor must be positive: experts have equal room")    # ExpertSort's capacity of 0 is another layout
        self.workers, self.vocab, self.width, self.hidden, self.blocks, self.tokens = workers, vocab, width, hidden, blocks, tokens
        self.experts, self.top, self.dtype, self.max_norm = experts, top, dtype, max_norm
        self.capacity = min(tokens, math.ceil(capacity_factor * tokens * top / experts))
        half = dtype == torch.float16
        self.loss_scale = loss_scale or (2.0 ** round(math.log2(min(tokens, 4096))) if half else 1.0)
        shape = dict(table=(vocab, width), pre=(width,), router=(experts, width), gate=(width,), post=(width,))
        matrices = dict(w_gate=(hidden, width), w_up=(hidden, width), w_down=(width, hidden))
        self.names, self.shapes = [(0, "table")], [shape["table"]]
        for b in range(blocks):
            for n in ("pre", "router", "gate", "post"):
                self.names.append((b, n))
                self.shapes.append(shape[n])
            for n, s in matrices.items():
                self.names += [(b, n, e) for e in range(experts)]
                self.shapes += [s] * experts
        self.names.append((blocks, "pre"))
        self.shapes.append((width,))
        numel = [int(np.prod(s)) for s in self.shapes]
        rng = np.random.default_rng(seed)
        first = []
        for (_, n, *_), s in zip(self.names, self.shapes):
            if len(s) == 2:
                first.append(rng.standard_normal(s).reshape(-1) / s[1] ** 0.5)
            else:
                first.append(np.full(s, 0.5 if n == "gate" else 1.0))
        x0 = np.broadcast_to(np.concatenate(first).astype(np.float32), (workers, sum(numel)))
        self.stream = stream if stream is not None else torch.cuda.current_stream(device)
        where = dict(device=device, stream=self.stream)
        with torch.cuda.stream(self.stream):
            self.ring = evg.Ring(x0, numel, lr=lr, momentum=momentum, grad_mode=evg.GRAD_BUFFER, **where, **ring_options)
            arena = self.ring.x
            self.grad = torch.zeros_like(arena)
            self.low = arena if dtype == torch.float32 else torch.empty_like(arena, dtype=dtype)
            self.low_grad = self.grad if dtype == torch.float32 else torch.zeros_like(self.low)
            self.params, self.grads = self._views(self.low), self._views(self.low_grad)
            rows = dict(workers=workers, dtype=dtype, **where)
            self.embed = nn.Embedding(vocab, width, max_tokens=tokens, scale=width ** 0.5, train=True, **rows)
            self.norm = nn.BlockNorm(width, max_rows=tokens, gate_rows=tokens, **rows)
            self.router = nn.Router(experts, top, workers=workers, max_tokens=tokens, dtype=torch.float32, **where)
            self.sort = nn.ExpertSort(experts, top, width, max_tokens=tokens, capacity=self.capacity, **rows)
            self.ffn = nn.GatedFFN(width, hidden, max_rows=self.capacity, activation=nn.ACTIVATIONS[activation], train=True, **rows)
            self.clip = nn.GradClip(numel, workers, dtype=dtype, out_dtype=torch.float32,
                                    nonfinite=nn.NONFINITE_ZERO if half else nn.NONFINITE_PASS, **where)
            self.updates = {}       # what makes a shape's updates; its tensors' momenta and places in the gradient
            if orthogonal:
                final = self._views(self.grad)
                for n, s in matrices.items():
                    if s not in self.updates:
                        self.updates[s] = (nn.Orthogonal(*s, matrices=workers, scale=orthogonal_scale * max(1.0, s[0] / s[1]) ** 0.5, **where), [])
                    for b in range(blocks):
                        self.updates[s][1].extend((torch.zeros(workers, *s, device=device), final[b, n, e]) for e in range(experts))
        self.stream.synchronize()
        self.k = 0

    def _slots(self, rows, e):
        """An expert's slots of all workers."""
        return rows[:, e * self.capacity:(e + 1) * self.capacity]

    def _real(self, numbers):
        """Which are in the vocabulary?"""
        return (numbers >= 0) & (numbers < self.vocab)

    def forward(self, tokens):
        """The last norm's rows [workers, tokens, width] of the ring's present parameters, and what the backward pass needs."""
        with self._ordered() as hand_over:
            if self.low is not self.ring.x:
                self.low.copy_(self.ring.x)
            p, kept = self.params, []
            residual = self.embed.forward(tokens, p[0, "table"])
            residual, normed = self.norm.forward(residual, pre=p[0, "pre"])
            for b in range(self.blocks):
                logits = torch.bmm(normed.float(), p[b, "router"].float().mT.contiguous()).masked_fill_(~self._real(tokens)[..., None], -math.inf)
                chosen, weights = self.router.forward(logits)
                rows, plan = self.sort.dispatch(normed, chosen)
                done, saved = torch.empty_like(rows), []
                for e in range(self.experts):
                    _, s = self.ffn.forward(self._slots(rows, e), p[b, "w_gate", e], p[b, "w_up", e], p[b, "w_down", e], out=self._slots(done, e), save=True)
                    saved.append(s)
                y = self.sort.combine(done, weights, plan)
                kept.append((residual, normed, logits, chosen, weights, rows, plan, done, saved, y))
                hand_over(residual, normed, logits, chosen, weights, rows, *plan, done, *saved, y)
                residual, normed = self.norm.forward(residual, y, gate=p[b, "gate"], post=p[b, "post"], pre=p[b + 1, "pre"])
            hand_over(residual, normed)
        return normed, kept

    def backward(self, d_out, tokens, kept):
        """Fills the gradient arena from the gradient of the rows; the table's is added to what is there from its use behind them."""
        with self._ordered():
            p, g = self.params, self.grads
            d_residual, d_normed = None, d_out
            for b in reversed(range(self.blocks)):
                residual, normed, logits, chosen, weights, rows, plan, done, saved, y = kept[b]
                d = self.norm.backward(d_residual, d_normed, residual, y, gate=p[b, "gate"], post=p[b, "post"], pre=p[b + 1, "pre"],
                                       out=dict(d_gate=g[b, "gate"], d_post=g[b, "post"], d_pre=g[b + 1, "pre"]))
                d_residual = d["d_residual"]
                d_done, d_weights = self.sort.combine_backward(d["d_branch"], done, weights, plan)
                d_rows = torch.empty_like(rows)
                for e in range(self.experts):
                    self.ffn.backward(self._slots(d_done, e), self._slots(rows, e), p[b, "w_gate", e], p[b, "w_up", e], p[b, "w_down", e], saved[e],
                                      dx=self._slots(d_rows, e), dw_gate=g[b, "w_gate", e], dw_up=g[b, "w_up", e], dw_down=g[b, "w_down", e])
                d_normed = self.sort.dispatch_backward(d_rows, plan)
                d_logits = self.router.backward(d_weights, logits, chosen)
                d_normed += torch.bmm(d_logits, p[b, "router"].float()).to(self.dtype)
                g[b, "router"].copy_(torch.bmm(d_logits.mT.contiguous(), normed.float()))
            d = self.norm.backward(d_residual, d_normed, kept[0][0], pre=p[0, "pre"], out=dict(d_pre=g[0, "pre"]))
            self.embed.backward(d["d_residual"], tokens, d_table=g[0, "table"], accumulate=True)

    def loss(self, out, tokens, target):
        """Each worker's mean cross entropy of the targets, the gradient of ``out`` (times the loss scale), and the table's, in its arena."""
        with self._ordered() as hand_over:
            real = self._real(tokens) & self._real(target)
            share = real / real.sum(1, keepdim=True).clamp(min=1)
            at = torch.where(real, target, 0).long()[..., None]
            table, rows = self.params[0, "table"].float(), out.float()
            logp = torch.log_softmax(torch.bmm(rows, table.mT.contiguous()), -1)
            loss = -(logp.gather(-1, at)[..., 0] * share).sum(1)
            d = logp.exp()
            d.scatter_add_(-1, at, torch.full(at.shape, -1.0, device=d.device))
            d *= (self.loss_scale * share)[..., None]
            self.grads[0, "table"].copy_(torch.bmm(d.mT.contiguous(), rows))
            d_out = torch.bmm(d, table).to(self.dtype)
            hand_over(loss, d_out)
        return loss, d_out

    def step(self, tokens, target):
        """One iteration on tokens and targets [workers, tokens]; each worker's loss and gradient norm, on the GPU."""
        with self._ordered() as hand_over:
            out, kept = self.forward(tokens)
            loss, d_out = self.loss(out, tokens, target)
            self.backward(d_out, tokens, kept)
            _, norm = self.clip.clip(self.low_grad, self.max_norm, out=self.grad, scale=1.0 / self.loss_scale)
            for op, tensors in self.updates.values():
                for m, grad in tensors:
                    op.update(grad, momentum=m, out=grad)
            self.ring.step(self.k, self.grad)
            self.k += 1
            hand_over(loss, norm)
        return loss, norm


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("workers", 4), ("vocab", 512), ("width", 128), ("hidden", 256), ("experts", 8), ("top", 2), ("blocks", 2), ("tokens", 128), ("steps", 40)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=("f32", "f16", "bf16"), default="bf16")
    ap.add_argument("--plain", action="store_true", help="SGD for the experts' matrices too")
    a = ap.parse_args(argv)
    dtype = dict(f32=torch.float32, f16=torch.float16, bf16=torch.bfloat16)[a.dtype]
    run = MixtureRing(a.workers, vocab=a.vocab, width=a.width, hidden=a.hidden, experts=a.experts, top=a.top, blocks=a.blocks, tokens=a.tokens, dtype=dtype,
                      orthogonal=not a.plain)
    gen = torch.Generator(device="cuda").manual_seed(1)
    after = torch.randperm(a.vocab, generator=gen, device="cuda")      # the language: each word has one that follows
    for k in range(a.steps):
        tokens = torch.randint(0, a.vocab, (a.workers, a.tokens), generator=gen, device="cuda")
        loss, norm = run.step(tokens, after[tokens])
        if k % 10 == 0 or k == a.steps - 1:
            print(f"step {k:4d}  loss {float(loss.mean()):.5f}  gradient norms {float(norm.min()):.4f} .. {float(norm.max()):.4f}", flush=True)
    st = run.ring.stats()
    print(f"{st['events_total']} of {st['regular_events']} messages sent, {st['bytes_sent'] / 1e6:.1f} MB")


if __name__ == "__main__":
    main()
