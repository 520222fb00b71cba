"""CPU-only checks of the paged cache's operators, beside test_cache_host.py: scales at their ends."""
import pytest

from paper_2506_09092_b200 import binding as B
from paper_2506_09092_b200 import build as libbuild
from test_cache_host import append, attn, shape


@pytest.fixture(scope="module", autouse=True)
def built():
    libbuild.build()


def test_a_scale_whose_product_is_no_number_is_refused():
    s = shape(scale=2.4e38)                            # log2 e times as much is above 3.4e38
    assert attn(s) == append(s) == B.ERR_INVALID_DIM and B.paged_attn_scratch_bytes(s) == 0
    for scale in (0.0, 1e-45, 2.0e38):
        assert attn(shape(scale=scale), q=None) == B.ERR_INVALID_POINTER
