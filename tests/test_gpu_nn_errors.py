"""An operator that could not be made leaves nothing behind that a later call would report as its own failure."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_calls_after_an_allocation_that_failed():
    from paper_2103_07454_amd import evg, nn
    op = nn.GradClip([8], 1)
    grad = torch.ones(1, op.pitch, device="cuda")
    with pytest.raises(evg.EvgError) as e:
        nn.GatedFFN(64, 1 << 20, max_rows=1 << 30)         # 2 PB of hidden values
    assert e.value.status == 3                              # EVG_ERR_OOM
    out, norm = op.clip(grad, 1.0)
    with pytest.raises(evg.EvgError):
        nn.GatedFFN(64, 1 << 20, max_rows=1 << 30)
    assert float(torch.ones(3, device="cuda").sum()) == 3.0
    assert abs(float(norm[0]) - 8 ** 0.5) < 1e-6
