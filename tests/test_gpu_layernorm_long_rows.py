"""Weight gradients of LayerNorm over rows of more than 16384 values: many rows, many columns."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def weight_gradients(dy, x, mean, rstd, dtype):
    rows, n = x.shape
    dg, db = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    size = B.layernorm_rows_bwd_scratch_bytes(rows, n)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    B.layernorm_rows_bwd(dy, x, None, mean, rstd, None, dg, db, rows, n, n, n, n, dtype, B.F32, scratch, size,
                         torch.cuda.current_stream())
    return dg, db


@pytest.mark.parametrize("rows,n,value", [(4000, 100000, 0.7), (4000, 100000, 1 / 3), (9000, 20000, 0.57)])
def test_roundings_that_all_point_one_way(rows, n, value):
    """A constant added again and again is rounded in the same direction each time, so a sum is off by the
    whole of its bound: m u of the terms' magnitudes for m additions one after the other, u = 2^-24.  A
    thread adds 32 rows, and then those sums, of which there are up to 32 (a part has at most 1024 rows here); the join
    adds up to 148 partial sums, at most 4 one after the other per lane, then 2 + 5 levels; xhat and its product bring
    3 roundings, the result's own 1."""
    dy = torch.full((rows, n), value, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.rand(rows, n, generator=gen, device="cuda")
    mean, rstd = torch.full((rows,), -0.5, device="cuda"), torch.full((rows,), 0.75, device="cuda")
    dg, db = weight_gradients(dy, x, mean, rstd, B.F32)
    bound = (32 + 32 + 4 + 7 + 3 + 1) * U * 1.001
    want = rows * dy[0, 0].double()
    assert float(((db.double() - want).abs() / want).max()) <= bound
    for c in range(0, n, 8192):                        # (every term is positive)
        part = slice(c, min(c + 8192, n))
        want = ((x[:, part].double() + 0.5) * 0.75 * dy[0, 0].double()).sum(0)
        assert float(((dg[part].double() - want).abs() / want).max()) <= bound


@pytest.mark.parametrize("rows", [1, 2])
def test_columns_whose_partial_rows_lie_beyond_32_bits(rows):
    """More than 2^30 columns: the second partial row's elements have indexes beyond 2^31.  Values whose
    products and sums are exact."""
    n = (1 << 30) + 1000
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, dy = (torch.empty(rows, n, dtype=torch.bfloat16, device="cuda").random_(-3, 4, generator=gen) for _ in range(2))
    mean, rstd = torch.zeros(rows, device="cuda"), torch.full((rows,), 0.5, device="cuda")
    dg, db = (torch.full((n,), 77.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    size = B.layernorm_rows_bwd_scratch_bytes(rows, n)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    B.layernorm_rows_bwd(dy, x, None, mean, rstd, None, dg, db, rows, n, n, n, n, B.BF16, B.BF16, scratch, size,
                         torch.cuda.current_stream())
    for c in range(0, n, 1 << 27):
        part = slice(c, min(c + (1 << 27), n))
        assert torch.equal(db[part], dy[:, part].sum(0))
        assert torch.equal(dg[part], (dy[:, part] * x[:, part] * 0.5).sum(0))
