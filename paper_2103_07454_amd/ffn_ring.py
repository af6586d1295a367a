"""Ring workers that train a stack of gated feed-forward blocks: the operators of ``nn`` and the ring's step together.

Every worker has its own copy of the parameters in the ring's arena and its own tokens.  A step runs, for all workers at once,

    forward     normed, y of each block: BlockNorm.forward, GatedFFN.forward
    backward    BlockNorm.backward, GatedFFN.backward, which write each parameter's gradient where the ring looks for it
    clipping    GradClip: each worker's gradient to at most ``max_norm``, into the 32-bit arena
    the ring    Ring.step: triggers, sends, averaging with the neighbours and momentum SGD

In 32 bits the operators read the ring's arena itself.  In 16 bits they read a rounded copy of it and fill a 16-bit gradient
arena, which clipping widens.  The gradients of float16 are those of ``loss_scale`` times the loss: the loss is a mean over a
worker's values, so the gradient of one of them would lie among the subnormals.  Clipping takes the scale back, and a worker whose
scaled gradient overflows sits the step out.

All work is on the stream that the object was made with.  ``forward``, ``backward`` and ``step`` may be called under any other: they
begin behind what the caller's stream has been given so far, and the caller's stream goes on behind them.

    python -m paper_2103_07454_amd.ffn_ring --workers 8 --width 512 --hidden 2048 --blocks 2 --tokens 256 --dtype bf16
"""
from __future__ import annotations

import argparse
import contextlib
import math

import numpy as np
import torch

from . import evg, nn

#: The tensors of a block and their shapes: the norm ahead of it, its three matrices, its gate for each channel, the norm behind it.
_BLOCK = ("pre", "w_gate", "w_up", "w_down", "gate", "post")


class FFNRing:
    def __init__(self, workers=4, *, width=64, hidden=192, blocks=2, tokens=32, dtype=torch.float32, activation="silu",
                 lr=0.05, momentum=0.9, max_norm=1.0, seed=0, loss_scale=None,
                 device="cuda:0", stream=None, **ring_options):
        self.workers, self.width, self.hidden, self.blocks, self.tokens = workers, width, hidden, blocks, tokens
        self.dtype, self.max_norm = dtype, max_norm
        half = dtype == torch.float16
        # An error of 1 becomes a gradient of about 1, or less where there are so many tokens that a weight's gradient, a sum over
        # them, would reach float16's 65504.  A power of two: taking it back is exact.
        self.loss_scale = loss_scale or (2.0 ** round(math.log2(width * min(tokens, 4096))) if half else 1.0)
        shape = dict(pre=(width,), w_gate=(hidden, width), w_up=(hidden, width), w_down=(width, hidden), gate=(width,), post=(width,))
        self.names = [(b, n) for b in range(blocks) for n in _BLOCK] + [(blocks, "pre")]      # the last norm has no block behind it
        self.shapes = [shape[n] for _, n in self.names]
        numel = [int(np.prod(s)) for s in self.shapes]
        rng = np.random.default_rng(seed)
        first = []
        for (_, n), s in zip(self.names, self.shapes):
            if len(s) == 2:
                first.append(rng.standard_normal(s).reshape(-1) / s[1] ** 0.5)
            else:
                first.append(np.full(s, 0.5 if n == "gate" else 1.0))
        x0 = np.broadcast_to(np.concatenate(first).astype(np.float32), (workers, sum(numel)))
        # The ring and the operators share one stream: what one writes the next reads.
        self.stream = stream if stream is not None else torch.cuda.current_stream(device)
        where = dict(device=device, stream=self.stream)
        with torch.cuda.stream(self.stream):
            self.ring = evg.Ring(x0, numel, lr=lr, momentum=momentum, grad_mode=evg.GRAD_BUFFER, **where, **ring_options)
            arena = self.ring.x
            self.grad = torch.zeros_like(arena)                                   # what the ring takes
            self.low = arena if dtype == torch.float32 else torch.empty_like(arena, dtype=dtype)
            self.low_grad = self.grad if dtype == torch.float32 else torch.zeros_like(self.low)
            self.params, self.grads = self._views(self.low), self._views(self.low_grad)
            self.norm = nn.BlockNorm(width, workers=workers, max_rows=tokens, dtype=dtype, gate_rows=tokens, **where)
            self.ffn = nn.GatedFFN(width, hidden, workers=workers, max_rows=tokens, dtype=dtype, activation=nn.ACTIVATIONS[activation],
                                   train=True, **where)
            self.clip = nn.GradClip(numel, workers, dtype=dtype, out_dtype=torch.float32,
                                    nonfinite=nn.NONFINITE_ZERO if half else nn.NONFINITE_PASS, **where)
        self.stream.synchronize()
        self.k = 0

    def _views(self, arena):
        """{(block, name): [workers, ...]} of an arena; a gate is [workers, 1, width], the row that all tokens share."""
        lay, out = self.ring.layout, {}
        for key, shape, off, n in zip(self.names, self.shapes, lay.offsets, lay.numel):
            v = arena[:, int(off):int(off) + int(n)]
            out[key] = v[:, None] if key[1] == "gate" else v.unflatten(1, shape) if len(shape) == 2 else v
        return out

    @contextlib.contextmanager
    def _ordered(self):
        """The block's work goes to the object's stream, between what the caller's has been given before and after.  Yields what hands
        tensors of the block to the caller: their memory is not used again before the caller's stream is done with them."""
        caller = torch.cuda.current_stream(self.stream.device)
        if caller == self.stream:
            yield lambda *tensors: None
            return
        self.stream.wait_stream(caller)
        try:
            with torch.cuda.stream(self.stream):
                yield lambda *tensors: [t.record_stream(caller) for t in tensors]
        finally:
            caller.wait_stream(self.stream)

    def forward(self, x):
        """The output [workers, tokens, width] of the ring's present parameters, and what the backward pass needs."""
        with self._ordered() as hand_over:
            if self.low is not self.ring.x:
                self.low.copy_(self.ring.x)
            p, kept = self.params, []
            residual, normed = self.norm.forward(x, pre=p[0, "pre"])
            for b in range(self.blocks):
                y, saved = self.ffn.forward(normed, p[b, "w_gate"], p[b, "w_up"], p[b, "w_down"], save=True)
                kept.append((residual, normed, y, saved))
                hand_over(*kept[-1])
                residual, normed = self.norm.forward(residual, y, gate=p[b, "gate"], post=p[b, "post"], pre=p[b + 1, "pre"])
            hand_over(normed)
        return normed, kept

    def backward(self, d_out, kept):
        """Fills the gradient arena from the gradient of the output."""
        with self._ordered():
            p, g = self.params, self.grads
            d_residual, d_normed = None, d_out
            for b in reversed(range(self.blocks)):
                residual, normed, y, saved = kept[b]
                d = self.norm.backward(d_residual, d_normed, residual, y, gate=p[b, "gate"], post=p[b, "post"], pre=p[b + 1, "pre"],
                                       out=dict(d_gate=g[b, "gate"], d_post=g[b, "post"], d_pre=g[b + 1, "pre"]))
                d_residual = d["d_residual"]
                d_normed, *_ = self.ffn.backward(d["d_branch"], normed, p[b, "w_gate"], p[b, "w_up"], p[b, "w_down"], saved,
                                                 dw_gate=g[b, "w_gate"], dw_up=g[b, "w_up"], dw_down=g[b, "w_down"])
            self.norm.backward(d_residual, d_normed, kept[0][0], pre=p[0, "pre"], out=dict(d_pre=g[0, "pre"]))

    def step(self, x, target):
        """One iteration on inputs and targets [workers, tokens, width]; each worker's loss and gradient norm, on the GPU."""
        with self._ordered() as hand_over:
            out, kept = self.forward(x)
            error = out.float() - target.float()
            self.backward((error / (error[0].numel() / self.loss_scale)).to(self.dtype), kept)
            _, norm = self.clip.clip(self.low_grad, self.max_norm, out=self.grad, scale=1.0 / self.loss_scale)
            self.ring.step(self.k, self.grad)
            self.k += 1
            loss = 0.5 * error.square().mean((1, 2))
            hand_over(loss, norm)
        return loss, norm


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("workers", 4), ("width", 256), ("hidden", 704), ("blocks", 2), ("tokens", 128), ("steps", 40)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=("f32", "f16", "bf16"), default="bf16")
    ap.add_argument("--max-norm", type=float, default=1.0)
    a = ap.parse_args(argv)
    dtype = dict(f32=torch.float32, f16=torch.float16, bf16=torch.bfloat16)[a.dtype]
    run = FFNRing(a.workers, width=a.width, hidden=a.hidden, blocks=a.blocks, tokens=a.tokens, dtype=dtype, max_norm=a.max_norm, lr=0.2)
    gen = torch.Generator(device="cuda").manual_seed(1)
    teacher = torch.randn(a.width, a.width, generator=gen, device="cuda") / a.width ** 0.5
    for k in range(a.steps):
        x = torch.randn(a.workers, a.tokens, a.width, generator=gen, device="cuda")
        loss, norm = run.step(x.to(dtype), torch.tanh(x @ teacher))
        if k % 10 == 0 or k == a.steps - 1:
            print(f"step {k:4d}  loss {float(loss.mean()):.5f}  gradient norms {float(norm.min()):.4f} .. {float(norm.max()):.4f}", flush=True)
    st = run.ring.stats()
    print(f"{st['events_total']} of {st['regular_events']} messages sent, {st['bytes_sent'] / 1e6:.1f} MB")


if __name__ == "__main__":
    main()
