"""CPU-only: results that lie over an operand with another pitch are refused before any CUDA call."""
import pytest

from paper_2506_09092_b200 import binding as B
from paper_2506_09092_b200 import build as libbuild

P, Q = 1 << 20, 1 << 24


@pytest.fixture(scope="module", autouse=True)
def built():
    libbuild.build()


@pytest.mark.parametrize("ldx,ldy", [(8, 16), (16, 8)])
def test_forward_over_its_input(ldx, ldy):
    assert B.layernorm_rows(P, None, None, P, None, None, 4, 8, ldx, ldy, B.BF16, B.F32, check=False) == B.ERR_INVALID_LD


@pytest.mark.parametrize("dx,lddx,lddy,ldx", [(P, 16, 8, 16), (Q, 16, 16, 8), (P, 8, 16, 8), (Q, 8, 8, 16)])
def test_backward_over_an_input(dx, lddx, lddy, ldx):
    st = B.layernorm_rows_bwd(P, Q, None, P + 4096, P + 8192, dx, None, None, 4, 8, lddy, ldx, lddx, B.BF16, B.F32,
                              None, 0, check=False)
    assert st == B.ERR_INVALID_LD
