"""Clipping at the ends of the bound's range: what never clips leaves every gradient as it is, and no finite gradient becomes NaN."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
         (torch.float16, torch.float32), (torch.float16, torch.float16)]
IDS = ["f32", "bf16-f32", "bf16", "f16-f32", "f16"]
#: One chunk of sums; more of them than a workgroup adds up for itself (a launch of its own does).
LISTS = [[10, 20], [5] * 600]


@pytest.fixture(scope="module")
def nn():
    from paper_2103_07454_amd import nn as m
    return m


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("numel", LISTS, ids=["few", "many"])
def test_an_infinite_bound_never_clips(nn, types, numel):
    dtype, out_dtype = types
    op = nn.GradClip(numel, 2, dtype=dtype, out_dtype=out_dtype)
    grad = torch.ones(2, op.pitch, dtype=dtype, device="cuda")
    grad[1, 3] = math.inf
    out, norm = op.clip(grad, math.inf, out=torch.ones(2, op.pitch, dtype=out_dtype, device="cuda"))
    assert torch.equal(out.to(dtype), grad) and norm[1] == math.inf
    out, _ = op.clip(grad, math.inf, out=torch.ones(2, op.pitch, dtype=out_dtype, device="cuda"), scale=0.5)
    assert float(out[1, 0]) == 0.5 and float(out[1, 3]) == math.inf
    grad[1, 3] = math.nan
    out, norm = op.clip(grad, math.inf)
    assert math.isnan(norm[1]) and math.isnan(out[1, 0]) and float(out[0, 0]) == 1.0
    out, _ = nn.GradClip(numel, 2, dtype=dtype, out_dtype=out_dtype, nonfinite=nn.NONFINITE_ZERO).clip(grad, math.inf)
    assert float(out[1, 0]) == 0.0 and float(out[1, 3]) == 0.0 and float(out[0, 0]) == 1.0


def test_an_infinite_bound_keeps_gradients_whose_norm_32_bits_do_not_hold(nn):
    grad = torch.full((1, 64), 3e38, device="cuda")
    out, norm = nn.GradClip([40], 1).clip(grad, math.inf)
    assert norm[0] == math.inf and torch.equal(out[:, :40], grad[:, :40])


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("numel", LISTS, ids=["few", "many"])
def test_no_gradient_and_no_bound(nn, types, numel):
    """0 / (0 + 0): a gradient of zeros stays one."""
    dtype, out_dtype = types
    op = nn.GradClip(numel, 2, dtype=dtype, out_dtype=out_dtype, eps=0.0)
    grad = torch.zeros(2, op.pitch, dtype=dtype, device="cuda")
    grad[1, 2] = 2.0
    out, norm = op.clip(grad, 0.0, out=torch.ones(2, op.pitch, dtype=out_dtype, device="cuda"))
    assert norm.tolist() == [0.0, 2.0] and float(out[:, :5].float().abs().max()) == 0.0
