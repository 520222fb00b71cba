"""The drawn token has to be the very one at the point drawn, unless the point lies within 2^-35 of the sum of a border, where 64-bit
sums of another order may fall on the other side: that is to be expected for about one in 2^35 / vocab tokens drawn."""
import pytest
import torch

from test_gpu_draft_verify import call, expect, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("b,n,vocab", [(40, 3, 511), (200, 2, 4097), (300, 1, 9000), (30, 3, 50001), (20, 2, 200000)])
def test_the_very_token_at_the_point(b, n, vocab, certain, dtype):
    p, q, drafts, u = inputs(b, n, vocab, dtype, 3 * vocab + n, certain)
    tokens, accepted = call(p, q, drafts, None, u, vocab, dtype)
    borders = 0
    for i, (a, _, may) in enumerate(expect(*(None if t is None else t.cpu() for t in (p, q, drafts, None, u)))):
        assert accepted[i].item() == a
        if len(set(may)) == 1:
            assert tokens[i, a].item() == may[0], i
        else:
            borders += 1
            assert tokens[i, a].item() in may, i
    assert borders <= 1
