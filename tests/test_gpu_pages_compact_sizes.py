"""Compaction of books of sizes around the limit of what a launch gets without asking for more shared memory."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
REPO = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

COMPACT = """
import sys
sys.path.insert(0, {repo!r})
import torch
from paper_2506_09092_b200 import binding as B
for pages in (391104, 391105, 393216, 393217):
    book = B.PageBook(pages, 2, 2, 10)
    book.lens[1] = 20
    at = torch.arange(10, device="cuda") * 7 + pages - 64
    book.table[1], book.refs[at] = at.int(), 1
    n = B.pages_compact_scratch_bytes(book)
    scratch, used = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.pages_compact(book, None, used, scratch, n, torch.cuda.current_stream())
    assert used.item() == 10 and book.table[1].tolist() == list(range(10)), pages
    assert book.refs.nonzero().flatten().tolist() == list(range(10)), pages
print("compacted")
"""


def test_compaction_by_a_process_that_has_not_compacted_a_larger_book():
    p = subprocess.run([sys.executable, "-c", COMPACT.format(repo=REPO)], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and "compacted" in p.stdout, p.stderr[-2000:]
