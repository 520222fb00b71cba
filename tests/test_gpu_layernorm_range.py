"""LayerNorm over rows at the ends of fp32's range: what include/cudallm_layers.h says of rows whose sums leave it."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,code", [(torch.float32, B.F32), (torch.bfloat16, B.BF16)])
@pytest.mark.parametrize("n", [40, 1000, 4096, 20000])
def test_rows_whose_sums_leave_the_range(n, dtype, code):
    x = torch.randn(5, n, device="cuda")
    x[1] *= 1e18                              # squares up to 2.5e37, their sum below 3.4e38 / n only for short rows
    x[2] *= 1e25                              # squares beyond fp32
    x[3] = 3e38                               # sum beyond fp32
    x = x.to(dtype)
    gamma, beta = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    B.layernorm_rows(x, gamma, beta, y, mean, rstd, 5, n, n, n, code, B.F32, 1e-5, torch.cuda.current_stream())
    if n == 40:                               # 40 values of 1e18: sum of squares 4e37
        d = x[1].double() - x[1].double().mean()
        want = d / torch.sqrt((d * d).mean()) * gamma.double() + beta.double()
        eps = torch.finfo(dtype).eps / 2
        # (40 additions and a dozen roundings of 2^-24, then the result's own)
        assert bool(((y[1].double() - want).abs() <= want.abs() * eps * 1.001 + 60 * 2.0 ** -24 * (want - beta).abs() + 1e-6).all())
    assert float(rstd[2]) == 0 and torch.equal(y[2], beta.to(dtype))
    assert bool(y[3].isnan().all())
    for row in (0, 4):
        d = x[row].double() - x[row].double().mean()
        assert abs(float(rstd[row]) - float(1 / torch.sqrt((d * d).mean() + 1e-5))) <= 1e-5 and bool(y[row].isfinite().all())
