"""How many pages a refused resize says are missing, whatever is asked for: also more than the book has."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B
from test_gpu_pages import Pair, ints

pytestmark = pytest.mark.gpu


def test_one_sequence_lacks_more_pages_than_there_are():
    p = Pair(8, 4, 4, 40)
    assert p.resize([0], [128]) == 24
    assert p.resize([1], [16]) == 0
    assert p.resize([0], [128]) == 28
    assert p.resize([0, 2, 1], [160, 160, 17]) == 40 + 40 + 1 - 4
    assert p.resize([0, 1], [160, 0]) == 32
    p.fork([1], [2])
    p.resize([1], [13])                                # its last page is shared, and no longer full
    assert p.resize([2, 1], [160, 14]) == 36 + 1 - 4
    assert p.resize([3], [161]) == -1


@pytest.mark.parametrize("entries", [3, 1024, 1025, 3000])
def test_many_sequences_lack_pages(entries):
    p = Pair(50, 2, entries, 400, pools=0)
    assert p.resize([1], [30]) == 0
    assert p.resize(None, [800] * entries) == entries * 400 - 15 - 35


def test_more_missing_pages_than_the_result_can_say():
    book = B.PageBook(8, 1, 3, 1 << 30)
    n = B.pages_resize_scratch_bytes(book, 3)
    scratch, result = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for want, missing in (([1 << 30, 0, 0], (1 << 30) - 8), ([1 << 30, 1 << 29, 5], (3 << 29) + 5 - 8), ([1 << 30] * 3, (1 << 31) - 1)):
        B.pages_resize(book, None, None, ints(want), 3, result, scratch, n, torch.cuda.current_stream())
        assert result.item() == missing and not book.lens.any() and not book.refs.any()
