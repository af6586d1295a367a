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
