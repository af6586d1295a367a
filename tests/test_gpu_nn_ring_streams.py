"""FFNRing on streams other than the default one: the ring, the operators and the work between them are in one order."""
import pytest
import torch

from test_gpu_nn_ring import data

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
SIZES = dict(width=64, hidden=192, tokens=64, lr=0.2)


def train(run, steps, seen=None):
    for k in range(steps):
        out = run.step(*data(run, k))
        if seen is not None:
            seen.append([v.clone() for v in out])
    torch.cuda.synchronize()
    return run.ring.state("x")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_everything_is_on_the_stream_that_is_given(dtype):
    from paper_2103_07454_amd import ffn_ring
    stream = torch.cuda.Stream()
    run = ffn_ring.FFNRing(3, dtype=dtype, stream=stream, **SIZES)
    assert all(part.stream == stream for part in (run.ring, run.norm, run.ffn, run.clip))
    want = train(ffn_ring.FFNRing(3, dtype=dtype, **SIZES), 4)
    with torch.cuda.stream(stream):
        got = train(run, 4)
    assert (got == want).all()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("made_on_its_own", [False, True], ids=["made on the default stream", "made on its own stream"])
def test_steps_from_another_stream(dtype, made_on_its_own):
    """Both streams are kept busy ahead of every step, so that work which did not wait would come early on either side."""
    from paper_2103_07454_amd import ffn_ring
    reference, seen, got = ffn_ring.FFNRing(3, dtype=dtype, **SIZES), [], []
    want = train(reference, 6, seen)
    run = ffn_ring.FFNRing(3, dtype=dtype, stream=torch.cuda.Stream() if made_on_its_own else None, **SIZES)
    busy = torch.randn(2048, 2048, device="cuda")
    torch.cuda.synchronize()
    caller = torch.cuda.Stream()
    for k in range(6):
        with torch.cuda.stream(caller):
            x, target = data(run, k)
        with torch.cuda.stream(run.stream):
            for _ in range(20):
                busy = (busy @ busy).mul_(1e-2).clamp_(-1, 1)      # the ring's stream is behind
        with torch.cuda.stream(caller):
            slow = torch.ones(2048, 2048, device="cuda")
            for _ in range(20):
                slow = (slow @ slow).clamp_(0, 1)                   # and so is the caller's: x comes late
            x.mul_(slow[:1, :1].to(x.dtype))
            loss, norm = run.step(x, target)
            x.zero_(), target.zero_()                               # the caller's tensors are its own again
            got.append([loss.clone(), norm.clone()])
            del x, target, loss, norm
    torch.cuda.synchronize()
    assert (run.ring.state("x") == want).all()
    assert all(torch.equal(a, b) for one, two in zip(seen, got) for a, b in zip(one, two))


def test_forward_and_backward_from_another_stream():
    from paper_2103_07454_amd import ffn_ring
    run = ffn_ring.FFNRing(3, dtype=torch.bfloat16, **SIZES)
    x, target = data(run, 0)
    out, kept = run.forward(x)
    run.backward(target.to(run.dtype), kept)
    want = out.clone(), run.low_grad.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        run.low_grad.zero_()
        out, kept = run.forward(x)
        run.backward(target.to(run.dtype), kept)
        assert torch.equal(out, want[0]) and torch.equal(run.low_grad, want[1])
