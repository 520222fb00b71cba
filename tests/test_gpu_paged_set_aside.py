"""Values that are not finite among the newest states, where the query rows do not fill the warps that they lie in: the rows that
see them take them, those before them and the other items do not, and the last item's rows end where the queries do (what lies
behind them is another tensor's)."""
import pytest
import torch

from paged_util import Cache, check, run
from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,group", [(5, 8), (33, 1), (3, 7), (43, 3), (65, 2), (2, 17)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("batch", [1, 3])
def test_of_the_last_item(batch, dim, rows, group):
    n = rows + 130
    c = Cache([n] * batch, rows, 2 * group, 2, dim, "bf16", 16, cols=3000, seed=rows)
    around = torch.full((c.q.numel() + 64 * 2 * group * dim,), float("nan"), dtype=c.q.dtype, device="cuda")
    q = around[:c.q.numel()].view(c.q.shape)
    q.copy_(c.q)
    c.q, last = q, batch - 1
    clean, _ = check(c)
    h = torch.finfo(c.q.dtype).eps / 2
    for bad in (float("nan"), float("inf"), float("-inf")):
        for back in {1, 2, rows // 2 + 1, rows}:
            page, row = c.at(last, n - back, 1)
            keep = c.v[page, row].clone()
            c.v[page, row, :, 3] = bad
            out = torch.full_like(c.q, 7.0)
            run(c, out)
            seen = rows - back                         # tokens from this one on see it
            want = torch.full((rows - seen, 2 * group), bad, dtype=out.dtype, device="cuda")
            assert torch.equal(out[last, seen:, :, 3].nan_to_num(9.0), want.nan_to_num(9.0))
            rest = [d for d in range(dim) if d != 3]
            # added in another order and from weights that are not rounded: each within h (|O| + sum p |v|)
            a, b = out[last][:, :, rest].float(), clean[last][:, :, rest].float()
            assert bool(((a - b).abs() <= 2.1 * h * (b.abs() + c.values[last].float().abs().max())).all())
            assert torch.equal(out[last, :seen], clean[last, :seen]) and torch.equal(out[:last], clean[:last])
            c.v[page, row] = keep
