"""The embeddings' gradient where one number has half of the tokens, or all of them: sums that go through hundreds of chunks."""
import pytest
import torch

import nn_experts_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,width", [(512, 40), (4096, 40), (16384, 40), (16399, 7), (40000, 300)], ids=lambda v: str(v))
@pytest.mark.parametrize("share", [0.5, 1.0], ids=["half", "all"])
def test_one_number_has_many_tokens(dtype, tokens, width, share):
    from paper_2103_07454_amd import nn
    V = 1000
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    ids = torch.randint(0, V, (2, tokens), generator=gen, device="cuda")
    ids[torch.rand(2, tokens, generator=gen, device="cuda") < share] = 17
    dy = (torch.randn(2, tokens, width, generator=gen, device="cuda") + 0.5).to(dtype)      # the common number's sum is far from 0
    op = nn.Embedding(V, width, workers=2, max_tokens=tokens, dtype=dtype, scale=0.5, train=True)
    got = op.backward(dy, ids)
    assert torch.equal(got, op.backward(dy, ids))
    for w in range(2):
        d = dy[w].double()
        common = ids[w] == 17

        def sums(v):
            total = torch.zeros(V, width, dtype=torch.float64, device="cuda").index_add_(0, ids[w][~common], v[~common])
            total[17] = v[common].sum(0)      # not by index_add_, whose additions to one row wait for each other
            return 0.5 * total

        value, size = sums(d), sums(d.abs())
        count = torch.bincount(ids[w], minlength=V).double()[:, None]
        bound = (count + 1) * ref.U32 * size
        off = (got[w].double() - value).abs()
        assert bool((off <= bound + ref.rounding(value.abs() + bound, dtype)).all())
        # Chunks of 16 are added up one by one, and then their sums: the common number's error is that of so few additions, not of one for each token.
        fewer = (16 + count[17] / 16 + 2) * ref.U32 * size[17]
        assert bool((off[17] <= fewer + ref.rounding(value[17].abs() + fewer, dtype)).all())
