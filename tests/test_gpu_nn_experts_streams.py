"""Calls of the operators for tokens, experts and orthogonal updates under another stream than their own run behind what their own has been given."""
import pytest
import torch

import test_gpu_nn_experts_graph as graph

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("few", [True, False], ids=["few", "many"])
def test_inputs_that_the_own_stream_still_has_to_write(few):
    """The tensors hold other numbers than those that the operators' stream is about to write, behind products that keep it busy: work on any other stream would begin
    at once and read the old ones."""
    own, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(own):
        fill, run = graph.passes(own, few)
        fill(1)
        want = [v.clone() for v in run()]
        fill(2)
        old = [v.clone() for v in run()]
    own.synchronize()
    # Every result tells the two apart; whole numbers of a few tokens may agree by chance.
    assert not any(torch.equal(a, b) for a, b in zip(want, old) if a.is_floating_point() or not few)
    busy = torch.randn(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    begin, end = torch.cuda.Event(), torch.cuda.Event()
    with torch.cuda.stream(own):
        for _ in range(10):
            busy @ busy
        begin.record()
        fill(1)
    with torch.cuda.stream(other):
        got = run()
        end.record(own)
        waiting = not begin.query()      # all calls were made while the own stream was still ahead of the new numbers
    own.synchronize()
    assert waiting, "the stream was not kept busy long enough for this to test anything"
    assert all(torch.equal(a, b) for a, b in zip(want, got))
