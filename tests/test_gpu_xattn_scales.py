"""Cross attention under tiny scales: keys times 2^100 under a scale times 2^-100 are the same scores, and multiplying by a power of two rounds
nothing, so the results are the same bits (the keys' gradient 2^-100 of itself)."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B
from test_gpu_xattn import operands, run_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q_rows,kv_rows,hq,hk,dim", [(1, 700, 8, 2, 64), (2, 9000, 4, 2, 128), (200, 300, 4, 2, 64), (130, 1500, 2, 1, 128)])
def test_tiny_scales_of_huge_scores(q_rows, kv_rows, hq, hk, dim):
    q, k, v, _ = operands(2, q_rows, kv_rows, hq, hk, dim, "bf16")
    scale, far = dim ** -0.5, 2.0 ** 100
    g = torch.Generator(device="cuda").manual_seed(3)
    do, out = torch.randn(q.shape, generator=g, device="cuda").bfloat16(), []
    for keys, s in ((k, scale), (k * far, scale / far)):
        o = torch.empty_like(q)
        lse = run_forward(q, keys, v, None, o, True, s)
        grads = [torch.empty_like(t) for t in (q, k, v)]
        shape = B.XattnShape.of(q, keys, v, o, s)
        n = B.xattn_bwd_scratch_bytes(shape)
        scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        B.xattn_bwd(shape, q, keys, v, None, o, lse, do, *grads, scratch, n, torch.cuda.current_stream())
        out.append((o, lse, grads[0], grads[2], grads[1].double() * (far if s < 1e-30 else 1.0)))
    for name, a, b in zip(("o", "lse", "dq", "dv"), *out):
        assert torch.equal(a, b), name
    # (what lies below bf16's normal range, 2^-126, is rounded to 2^-134)
    assert bool(((out[0][4] - out[1][4]).abs() <= 2.0 ** -134 * far).all())


def test_a_scale_of_zero_evens_out_huge_scores():
    for q_rows in (1, 200):
        q, k, v, _ = operands(1, q_rows, 400, 2, 1, 64, "bf16")
        o, same = torch.empty_like(q), torch.empty_like(q)
        run_forward(q, k, v, None, same, False, 0.0)
        run_forward(q, k * 2.0 ** 110, v, None, o, False, 0.0)
        # weights of 1 to within 2^-20, each then rounded to bf16 (to 1 or one step below), against weights of 1
        assert bool(((o.float() - same.float()).abs() <= 2.0 ** -7 * v.float().abs().mean(1, keepdim=True) + 2.0 ** -7 * same.float().abs()).all())
