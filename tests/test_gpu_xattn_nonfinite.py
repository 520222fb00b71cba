"""A value that is not finite reaches every row that sees it, however the keys are split and however little
the row's probabilities leave of it (0 x inf is no number, as in one pass over the keys)."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu


def attend(q, k, v, lens=None):
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[0], q.shape[2], q.shape[1], device="cuda")
    shape = B.XattnShape.of(q, k, v, out)
    n = B.xattn_fwd_scratch_bytes(shape)
    scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    B.xattn_fwd(shape, q, k, v, lens, out, lse, scratch, n, torch.cuda.current_stream())
    assert B.device_status(torch.cuda.current_stream())[0] == B.OK
    return out, lse, n


# single tokens in one part, in a cluster's parts, in parts joined by a second launch; longer queries in one part
# (as many heads as leave the keys whole) and in parts
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_rows,heads,states,second_launch", [(1, 1, 200, False), (1, 1, 1500, False), (1, 1, 20000, True),
                                                               (40, 150, 1500, False), (40, 1, 5000, True)])
def test_an_infinity_behind_a_vanishing_weight(q_rows, heads, states, second_launch, dim, dtype):
    gen = torch.Generator(device="cuda").manual_seed(7)
    q = torch.ones(1, q_rows, heads, dim, device="cuda", dtype=dtype)
    k = torch.zeros(1, states, heads, dim, device="cuda", dtype=dtype)
    # scores of 0 in front, of scale x dim x (-400 / sqrt(dim)) = -400 behind: exp of that is 0 in fp32
    k[:, states // 2:] = -400.0 / dim ** 0.5
    v = torch.randn(1, states, heads, dim, generator=gen, device="cuda").to(dtype)
    clean, lse, n = attend(q, k, v)
    assert (n > 0) == second_launch and bool(clean.isfinite().all())
    for bad in (float("inf"), float("nan")):
        w = v.clone()
        w[0, states - 3, 0, 5] = bad
        out, same_lse, _ = attend(q, k, w)
        assert not bool(out[0, :, 0, 5].isfinite().any())
        others = torch.ones_like(out, dtype=torch.bool)
        others[0, :, 0, 5] = False
        assert torch.equal(out[others], clean[others]) and torch.equal(lse, same_lse)
        # (behind an item's states it is not seen)
        lens = torch.tensor([states - 3], dtype=torch.int32, device="cuda")
        assert bool(attend(q, k, w, lens)[0].isfinite().all())
