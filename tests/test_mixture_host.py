"""The parts of MixtureRing that are torch's own, on the CPU."""
import contextlib

import pytest
import torch

from paper_2103_07454_amd import mixture_ring


def run_without_a_ring(vocab, width, workers):
    """What ``loss`` needs, and no more."""
    gen = torch.Generator().manual_seed(0)
    run = object.__new__(mixture_ring.MixtureRing)
    run.vocab, run.dtype, run.loss_scale = vocab, torch.float32, 1.0
    run.params = {(0, "table"): torch.randn(workers, vocab, width, generator=gen)}
    run.grads = {(0, "table"): torch.zeros(workers, vocab, width)}
    run._ordered = lambda: contextlib.nullcontext(lambda *tensors: None)
    return run, torch.randn(workers, 6, width, generator=gen)


@pytest.mark.parametrize("kind", [torch.int64, torch.int32], ids=["int64", "int32"])
def test_numbers_outside_the_vocabulary_have_no_loss(kind):
    """A gather at a number that the table does not have ends the process on a GPU; here it raises."""
    run, out = run_without_a_ring(5, 3, 2)
    tokens = torch.tensor([[0, 1, 2, 3, 4, 0], [4, 3, 2, 1, 0, 0]], dtype=kind)
    target = torch.tensor([[1, 2, -1, -1, 0, -1], [-1, -1, -1, -1, -1, -1]], dtype=kind)
    tokens[0, 4] = -1
    want, d = run.loss(out, tokens, target)
    table = run.grads[0, "table"].clone()
    tokens[0, 4] = 5
    target[0, 2], target[0, 3], target[0, 5] = 5, 2 ** 31 - 1, -7
    target[1] = 100
    got, d2 = run.loss(out, tokens, target)
    assert torch.equal(got, want) and torch.equal(d, d2) and torch.equal(table, run.grads[0, "table"])
    logp = torch.log_softmax(out[0] @ run.params[0, "table"][0].T, -1)
    assert torch.allclose(want, torch.stack([-(logp[0, 1] + logp[1, 2]) / 2, torch.zeros(())]), rtol=1e-5)
    assert bool((d[0, 2:] == 0).all()) and bool((d[1] == 0).all())


@pytest.mark.parametrize("factor", [0, 0.0, -1.0, float("nan")])
def test_experts_without_room_are_refused(factor):
    """A capacity of 0 would be ExpertSort's packed rows, of which no expert would get any."""
    with pytest.raises(ValueError, match="capacity_factor"):
        mixture_ring.MixtureRing(2, capacity_factor=factor)
