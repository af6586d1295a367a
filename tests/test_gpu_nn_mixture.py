"""Tokens, experts and orthogonal updates together, as ring workers train with them: the gradients and updates that reach the ring."""
import numpy as np
import pytest
import torch

import nn_experts_reference as ref
import nn_reference

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
SIZES = [dict(vocab=50, width=64, hidden=96, experts=4, tokens=70), dict(vocab=11, width=36, hidden=50, experts=5, top=3, tokens=9, capacity_factor=0.8)]


def data(run, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens = torch.randint(0, run.vocab, (run.workers, run.tokens), generator=gen, device="cuda")
    tokens[:, -2:] = -1                                     # padding
    return tokens, torch.randint(0, run.vocab, (run.workers, run.tokens), generator=gen, device="cuda")


def reference_gradient(run, tokens, target, kept):
    """Each worker's gradient in 64 bits, by differentiating the model as it is defined, with the experts and slots that the run took."""
    lay, arena, grads = run.ring.layout, run.low.double().cpu(), []
    unit = lambda z: z / torch.sqrt(z.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    for w in range(run.workers):
        p = {}
        for key, shape, off, n in zip(run.names, run.shapes, lay.offsets, lay.numel):
            p[key] = arena[w, int(off):int(off) + int(n)].reshape(shape).clone().requires_grad_()
        ids = tokens[w].cpu()
        r = run.width ** 0.5 * p[0, "table"][ids.clamp(min=0)] * (ids >= 0)[:, None]
        for b in range(run.blocks):
            chosen, slot = kept[b][3][w].cpu().long(), kept[b][6].slot[w].cpu()
            h = unit(r) * p[b, "pre"]
            weight = torch.softmax((h @ p[b, "router"].t()).gather(-1, chosen.clamp(min=0)), -1) * (slot >= 0)
            y = torch.zeros_like(r)
            for e in range(run.experts):
                out = (nn_reference.act("silu", h @ p[b, "w_gate", e].t())[0] * (h @ p[b, "w_up", e].t())) @ p[b, "w_down", e].t()
                y = y + (weight * (chosen == e)).sum(-1, keepdim=True) * out
            r = r + p[b, "gate"] * (unit(y) * p[b, "post"])
        out = unit(r) * p[run.blocks, "pre"]
        loss = torch.nn.functional.cross_entropy((out @ p[0, "table"].t())[ids >= 0], target[w].cpu()[ids >= 0])      # padding has none
        grads.append(torch.cat([g.reshape(-1) for g in torch.autograd.grad(loss, [p[key] for key in run.names])]))
    return torch.stack(grads)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("sizes", SIZES, ids=["whole", "odd, with entries left out"])
def test_gradients_that_reach_the_ring(dtype, sizes):
    from paper_2103_07454_amd import mixture_ring
    run = mixture_ring.MixtureRing(3, dtype=dtype, max_norm=1e9, orthogonal=False, **sizes)
    for k in range(2):
        tokens, target = data(run, k)
        out, kept = run.forward(tokens)
        want = reference_gradient(run, tokens, target, kept)      # of the parameters ahead of the step
        run.step(tokens, target)
        got = torch.from_numpy(run.ring.layout.unpad(run.grad.cpu().numpy())).double()
        off = (got - want).norm(dim=1) / want.norm(dim=1)
        print(f"[mixture] {dtype} step {k}: gradients off by {off.max() / nn_reference.UNIT[dtype]:.2f} units", flush=True)
        # Some twelve tensors of a block and pass are rounded to the type, each independently, in two blocks: their errors add up to at most fifty
        # units of the whole, and the norms and softmaxes that they pass double that at most.
        assert float(off.max()) <= 100 * nn_reference.UNIT[dtype] * (4 if dtype == torch.float32 else 1)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_updates_that_reach_the_ring(dtype):
    from paper_2103_07454_amd import mixture_ring
    plain = mixture_ring.MixtureRing(3, dtype=dtype, orthogonal=False, max_norm=0.5, **SIZES[0])
    run = mixture_ring.MixtureRing(3, dtype=dtype, orthogonal_scale=0.3, max_norm=0.5, **SIZES[0])
    tokens, target = data(run, 0)
    plain.step(tokens, target)
    run.step(tokens, target)
    lay, old, new = run.ring.layout, plain.grad.double().cpu(), run.grad.double().cpu()
    for key, shape, off, n in zip(run.names, run.shapes, lay.offsets, lay.numel):
        part = slice(int(off), int(off) + int(n))
        for w in range(3):
            if len(key) < 3:
                assert torch.equal(new[w, part], old[w, part])
                continue
            g = old[w, part].reshape(shape)
            _, u = ref.momentum(g, torch.zeros_like(g), 0.95, True)
            want, bound = ref.orthogonal(u, torch.float32, scale=0.3 * max(1.0, shape[0] / shape[1]) ** 0.5)
            assert float((new[w, part].reshape(shape) - want).norm()) <= bound


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_steps_from_another_stream_and_on_a_stream_of_its_own(dtype):
    from paper_2103_07454_amd import mixture_ring
    reference, seen = mixture_ring.MixtureRing(3, dtype=dtype, **SIZES[0]), []
    for k in range(4):
        loss, norm = reference.step(*data(reference, k))
        assert torch.isfinite(loss).all() and torch.isfinite(norm).all()
        seen.append((loss.clone(), norm.clone()))
    torch.cuda.synchronize()
    run = mixture_ring.MixtureRing(3, dtype=dtype, stream=torch.cuda.Stream(), **SIZES[0])
    assert all(part.stream == run.stream for part in (run.ring, run.embed, run.norm, run.router, run.sort, run.ffn, run.clip, *(op for op, _ in run.updates.values())))
    busy, caller = torch.randn(2048, 2048, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    for k in range(4):
        with torch.cuda.stream(run.stream):
            busy @ busy
        with torch.cuda.stream(caller):
            busy @ busy
            loss, norm = run.step(*data(run, k))
            assert torch.equal(loss, seen[k][0]) and torch.equal(norm, seen[k][1])
    torch.cuda.synchronize()
    assert np.array_equal(run.ring.state("x"), reference.ring.state("x"))


def test_command(capsys):
    from paper_2103_07454_amd import mixture_ring
    mixture_ring.main(["--workers", "3", "--vocab", "40", "--width", "64", "--hidden", "64", "--experts", "4", "--tokens", "16", "--steps", "3"])
    assert "messages sent" in capsys.readouterr().out
