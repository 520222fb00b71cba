"""Attention over pages where the split over the GPU is at its ends: very many parts of one item, very many row tiles,
calls side by side, first calls that are captured.  (Tolerances as in paged_util.)"""
import os
import subprocess
import sys
import threading

import pytest
import torch

from paged_util import Cache, check, run
from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu
REPO = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("rows,group,page_rows", [(1, 1, 16), (2, 8, 16), (1, 16, 7), (5, 8, 24), (3, 10, 24), (5, 8, 16), (1, 100, 64)])
@pytest.mark.parametrize("dim", [64, 128])
def test_one_item_in_many_parts(rows, group, page_rows, dim):
    check(Cache([33333], rows, group, 1, dim, "bf16", page_rows, seed=dim + rows))


@pytest.mark.parametrize("rows,group", [(1, 4), (4, 8)])
def test_parts_without_states(rows, group):
    """Most of a long sequence's pages are not there: parts of it have nothing to add, whole stretches of them."""
    c = Cache([30000, 20000], rows, 2 * group, 2, 128, "bf16", 16)
    absent = []
    for i, keep in enumerate(([5, 900, 1874], [1249])):
        gone = [p for p in range(c.table.shape[1]) if p not in keep]
        c.table[i, gone] = -1
        absent.append([s for s in range(c.lens_host[i]) if s // 16 not in keep])
    check(c, absent=absent)
    c.table[1] = -1
    out, lse = check(c, absent=[absent[0], list(range(20000))])
    assert not out[1].any() and bool((lse[1] == float("-inf")).all())


@pytest.mark.parametrize("rows,group", [(1, 4), (4, 8)])
def test_a_part_that_is_no_number(rows, group):
    c = Cache([30000, 20000], rows, 2 * group, 2, 64, "bf16", 16)
    clean, bad = torch.empty_like(c.q), torch.empty_like(c.q)
    run(c, clean)
    for where in (0, 12345, 29990):
        page, row = c.at(0, where, 1)
        for what, dims in ((c.v, [3]), (c.k, list(range(64)))):
            keep = what[page, row].clone()
            what[page, row, 1, 3] = float("nan")
            run(c, bad)
            hot = torch.zeros_like(bad, dtype=torch.bool)
            hot[0, :, group:, dims] = True
            assert bool(bad[hot].isnan().all()) and torch.equal(bad[~hot], clean[~hot])
            what[page, row] = keep


@pytest.mark.parametrize("lens,rows,hq,hk,dim", [([3000], 3000, 8, 1, 64), ([900, 700, 10, 0, 650], 700, 8, 2, 128),
                                                  ([1500, 1500, 1400], 1300, 3, 1, 40)])
@pytest.mark.parametrize("page_rows", [16, 24])
def test_many_row_tiles(lens, rows, hq, hk, dim, page_rows):
    check(Cache(lens, rows, hq, hk, dim, "bf16", page_rows, seed=rows, news=[min(rows, n) for n in lens]))


def test_a_prompt_in_pieces_is_the_prompt():
    """The same tokens in one call and in calls of unequal numbers of them, over pages that are filled already: within the
    rounding of the probabilities, which other tiles may round against other maxima."""
    c = Cache([600], 600, 8, 2, 64, "bf16", 16)
    whole, _ = check(c)
    first = 0
    for n in (1, 16, 200, 383):
        q = c.q[:, first:first + n].contiguous()
        out = torch.empty_like(q)
        shape = B.PagedShape.of(q, c.k, c.v, out, c.table)
        size = B.paged_attn_scratch_bytes(shape)
        scratch = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        first += n
        lens = torch.tensor([first], dtype=torch.int32, device="cuda")
        B.paged_attn(shape, q, c.k, c.v, c.table, lens, None, None, out, None, scratch, size, torch.cuda.current_stream())
        a, b = out.float(), whole[:, first - n:first].float()
        # each is within h (|O| + sum p |v|) and the small terms of the formula
        assert bool(((a - b).abs() <= 2 * 1.1 * 2.0 ** -8 * (b.abs() + c.values[0].float().abs().max())).all())


def enqueue(c, out, scratch, stream):
    shape = c.shape(out)
    B.paged_attn(shape, c.q, c.k, c.v, c.table, c.lens, None, None, out, None, scratch, B.paged_attn_scratch_bytes(shape), stream)


def test_tiles_side_by_side():
    """Two calls of the kernel that takes all of an SM, over and over on two streams, one of them as a graph."""
    caches = [Cache([900, 1500, 20], 6, 32, 2, 128, "bf16", 16, cols=400, seed=1),
              Cache([3000] * 4, 9, 32, 4, 64, "fp16", 64, cols=400, seed=2)]
    want = [torch.empty_like(c.q) for c in caches]
    for c, w in zip(caches, want):
        run(c, w)
    outs = [torch.empty_like(w) for w in want]
    scr = [torch.full((B.paged_attn_scratch_bytes(c.shape(o)) + 64,), 0xFF, dtype=torch.uint8, device="cuda") for c, o in zip(caches, outs)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        enqueue(caches[0], outs[0], scr[0], torch.cuda.current_stream())
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(a):
            graph.replay()
        enqueue(caches[1], outs[1], scr[1], b)
    torch.cuda.synchronize()
    assert B.device_status(torch.cuda.current_stream())[0] == B.OK
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_host_threads():
    caches = [Cache([500 + 100 * i, 20], 1 + 4 * (i % 2), 16, 2, 64, "bf16", 16, seed=i) for i in range(4)]
    want = [torch.empty_like(c.q) for c in caches]
    for c, w in zip(caches, want):
        run(c, w)
    outs, torn = [torch.empty_like(w) for w in want], []
    torch.cuda.synchronize()

    def work(c, o):
        try:
            s = torch.cuda.Stream()
            scratch = torch.full((B.paged_attn_scratch_bytes(c.shape(o)) + 64,), 0xFF, dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            for _ in range(30):
                enqueue(c, o, scratch, s)
            s.synchronize()
        except Exception as e:                         # noqa: BLE001
            torn.append(e)
    threads = [threading.Thread(target=work, args=x) for x in zip(caches, outs)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not torn
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


FIRST = """
import sys
sys.path[:0] = [{repo!r}, {repo!r} + "/tests"]
import torch
from paged_util import Cache, check
from paper_2506_09092_b200 import binding as B
caches = [Cache([300, 70], 1, 8, 2, 64, "bf16", 16), Cache([40000], 1, 8, 2, 128, "bf16", 16), Cache([2000, 9], 6, 32, 2, 128, "fp16", 16)]
outs = [torch.full_like(c.q, 7) for c in caches]
graph, scratch = torch.cuda.CUDAGraph(), []
with torch.cuda.graph(graph):
    for c, o in zip(caches, outs):
        shape = c.shape(o)
        n = B.paged_attn_scratch_bytes(shape)
        scratch.append(torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))
        B.paged_attn(shape, c.q, c.k, c.v, c.table, c.lens, None, None, o, None, scratch[-1], n, torch.cuda.current_stream())
    book = B.PageBook(70000, 16, 4, 10)
    slots = torch.arange(4, dtype=torch.int32, device="cuda")
    need = max(B.pages_resize_scratch_bytes(book, 4), B.pages_fork_scratch_bytes(book, 4), B.pages_compact_scratch_bytes(book))
    own = torch.empty(need, dtype=torch.uint8, device="cuda")
    lens = torch.full((4,), 33, dtype=torch.int32, device="cuda")
    s = torch.cuda.current_stream()
    B.pages_resize(book, None, None, lens, 2, None, own, need, s)
    B.pages_fork(book, slots, slots + 2, 2, own, need, s)
    B.pages_compact(book, None, None, own, need, s)
graph.replay()
torch.cuda.synchronize()
for c, o in zip(caches, outs):
    assert torch.equal(check(c)[0], o)
assert book.lens.tolist() == [33] * 4 and book.refs[:7].tolist() == [2] * 6 + [0]
print("as captured")
"""


def test_first_calls_of_a_process_are_captured():
    p = subprocess.run([sys.executable, "-c", FIRST.format(repo=REPO)], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and "as captured" in p.stdout, p.stderr[-2000:]


@pytest.mark.parametrize("rows,group,hk,dim", [(1, 1, 400, 64), (3, 8, 200, 64), (2, 10, 160, 128), (1, 30, 300, 40)])
def test_more_key_heads_than_shares(rows, group, hk, dim):
    """Each CTA takes all of a key head's keys: nothing is left in parts, and no room is asked for them."""
    c = Cache([700, 0, 33, 130, 1], rows, group * hk, hk, dim, "bf16", 16, cols=3000)
    assert B.paged_attn_scratch_bytes(c.shape(torch.empty_like(c.q))) <= 16 * hk
    check(c)


@pytest.mark.parametrize("rows,group", [(1, 4), (6, 8)])
def test_the_same_slot_twice(rows, group):
    """Items may look at one sequence side by side: its states are read, nothing of it is written."""
    c = Cache([500, 90, 33], rows, 2 * group, 2, 64, "bf16", 16)
    q = torch.cat([c.q, c.q.flip(0)])
    slot_of = torch.tensor([0, 1, 2, 0, 1, 0], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    shape = B.PagedShape.of(q, c.k, c.v, out, c.table)
    n = B.paged_attn_scratch_bytes(shape)
    scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    B.paged_attn(shape, q, c.k, c.v, c.table, c.lens, slot_of, None, out, None, scratch, n, torch.cuda.current_stream())
    alone = torch.empty_like(q)
    for i, w in enumerate(slot_of.tolist()):
        one, at = q[i:i + 1], slot_of[i:i + 1]
        shape = B.PagedShape.of(one, c.k, c.v, alone[i:i + 1], c.table)
        n = B.paged_attn_scratch_bytes(shape)
        scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        B.paged_attn(shape, one, c.k, c.v, c.table, c.lens, at, None, alone[i:i + 1], None, scratch, n, torch.cuda.current_stream())
        a, b = out[i].float(), alone[i].float()                # (the split may differ: each within h (|O| + sum p |v|))
        assert bool(((a - b).abs() <= 2 * 1.1 * 2.0 ** -8 * (b.abs() + c.values[w].float().abs().max())).all())


@pytest.mark.parametrize("values", [8, 40, 5000])
def test_one_page_copied_to_several(values):
    pool = torch.randn(9, values, device="cuda").bfloat16()
    want = pool.clone()
    src, dst = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([5, 5, 5, 2], [1, 8, 0, 3]))
    want[[1, 8, 0]], want[3] = pool[5].clone(), pool[2].clone()
    B.pages_copy(B.page_pools([pool]), src, dst, 4, torch.cuda.current_stream())
    assert torch.equal(pool, want)
