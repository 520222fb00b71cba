"""Attention of the newest tokens over their sequence's pages, and appending to them."""
import ctypes

import pytest
import torch

from paged_util import Cache, cdiv, check, run
from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout,page_rows", [("rows", 16), ("heads", 64), ("joint", 7), ("padded", 1), ("rows", 100), ("heads", 24)])
@pytest.mark.parametrize("rows,hq,hk,dim", [(1, 4, 4, 64), (1, 8, 1, 128), (3, 8, 2, 40), (5, 16, 2, 128), (2, 6, 3, 8), (9, 8, 1, 72)])
def test_lengths_and_layouts(dtype, layout, page_rows, rows, hq, hk, dim):
    """Lengths around the ends of pages and tiles, shorter than the new tokens, none at all."""
    lens = [300, 0, 1, 16, 17, 127, 128, 129, 64, rows, max(rows - 1, 0), 1000]
    check(Cache(lens, rows, hq, hk, dim, dtype, page_rows, layout, seed=page_rows + rows))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,group", [(1, 1), (1, 16), (4, 4), (4, 8), (8, 8), (1, 40)])
@pytest.mark.parametrize("batch,kv_heads,cols", [(1, 1, 4), (1, 1, 4000), (3, 2, 60), (20, 8, 40), (200, 1, 20), (300, 2, 10)])
def test_splits(batch, kv_heads, cols, rows, group, dim):
    """Few and many items, wide and narrow tables: clusters of all sizes and equal shares, up to three items a thread."""
    page_rows = 16
    top = min(cols * page_rows, 20000 // batch + 40)
    lens = [max(0, top - (i * top) // max(batch - 1, 1) - (i % 3)) for i in range(batch)]
    check(Cache(lens, rows, kv_heads * group, kv_heads, dim, "bf16", page_rows, cols=cols, seed=batch))


@pytest.mark.parametrize("group", [1, 8])
@pytest.mark.parametrize("rows", [1, 6])
def test_one_long_sequence(rows, group):
    check(Cache([40001, 5], rows, 2 * group, 2, 128, "bf16", 32, "rows", spread=3.0))


def test_padding_slots_and_new_lens():
    lens = [90, 40, 200, 7, 33, 64]
    c = Cache(lens, 4, 8, 2, 64, "fp16", 16, "rows", slots=[5, -1, 0, 3, 2, 1], news=[4, 2, 0, 1, 9, -3], seed=3)
    check(c)
    c.slot_of[2] = len(c.lens) + 3                     # behind the last slot: not there
    c.where[2] = len(c.lens) + 3
    check(c)


@pytest.mark.parametrize("cols", [None, 3000])
@pytest.mark.parametrize("rows", [40, 300])
def test_a_prompt(rows, cols):
    """Many more rows than a tile: every token sees exactly its own past."""
    check(Cache([rows, rows + 77, rows - 13], rows, 6, 2, 64, "bf16", 16, cols=cols))


@pytest.mark.parametrize("rows,group", [(2, 2), (2, 20), (9, 8)])
@pytest.mark.parametrize("cols", [None, 2000])
def test_pages_that_are_not_there_are_left_out(cols, rows, group):
    c = Cache([100, 64, 33, 16, 300], rows, 2 * group, 2, 64, "bf16", 16, cols=cols)
    absent = [range(16, 32), range(0, 64), range(32, 33), [], [*range(0, 128), *range(288, 300)]]
    c.table[0, 1] = -1
    c.table[1, :4] = c.k.shape[0]
    c.table[2, 2] = 1 << 30
    c.table[4, :8] = -7
    c.table[4, 18] = -1
    out, lse = check(c, absent=[list(a) for a in absent])
    assert not out[1].any() and bool((lse[1] == float("-inf")).all())


@pytest.mark.parametrize("page_rows", [8, 16, 32, 64, 128, 256, 384, 24])
@pytest.mark.parametrize("layout", ["rows", "heads", "joint", "padded"])
@pytest.mark.parametrize("dim", [40, 64, 128])
def test_many_rows_on_a_key_head(dim, layout, page_rows):
    """Pages of all sizes that fill a tile, and one that does not."""
    lens = [1000, 127, 0, 128, 129, 5, 400, 4000]
    check(Cache(lens, 6, 16, 2, dim, "bf16", page_rows, layout, cols=cdiv(40000, page_rows), seed=page_rows))


@pytest.mark.parametrize("batch,rows,hq,hk,dim", [(40, 3, 16, 2, 64), (3, 5, 128, 1, 128), (300, 2, 10, 1, 64), (1, 700, 3, 1, 128), (150, 17, 2, 2, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_many_rows_equal_shares(dtype, batch, rows, hq, hk, dim):
    """Shares that begin and end anywhere in an item; several row tiles; more items than threads that count them."""
    lens = [max(0, 2000 // (1 + batch // 20) + rows - 37 * (i % 50)) for i in range(batch)]
    news = [(i * 7) % (rows + 1) for i in range(batch)]
    check(Cache(lens, rows, hq, hk, dim, dtype, 16, cols=1000, seed=batch, news=news))


def test_lengths_beyond_the_table_and_below_zero():
    c = Cache([64, 64], 1, 4, 2, 64, "bf16", 16)
    c.lens[0], c.lens[1] = 1 << 30, -5
    c.lens_host[1], c.keys[1], c.values[1] = 0, c.keys[1][:0], c.values[1][:0]
    check(c)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 8])
@pytest.mark.parametrize("cols", [None, 3000])
def test_values_that_are_not_finite_reach_those_who_see_them(cols, group, dim, dtype):
    """Infinities and NaN in the keys and values of the newest tokens: a token before them is as if they were not
    there."""
    rows, n = 5, 150
    c = Cache([n, n, n, n], rows, 2 * group, 2, dim, dtype, 16, cols=cols, seed=group)
    clean = torch.empty_like(c.q)
    run(c, clean)
    for bad in (float("nan"), float("inf"), float("-inf")):
        for what in (c.k, c.v):
            for i, back in ((0, 1), (1, 2), (2, 4)):           # the last, the one before it, the fourth from the end
                page, row = c.at(i, n - back, 1)
                keep = what[page, row].clone()
                what[page, row, :, 3] = bad
                out = torch.empty_like(c.q)
                lse = torch.empty(4, 2 * group, rows, device="cuda")
                run(c, out, lse)
                seen = rows - back                                    # tokens from this one on see it
                if what is c.v and bad == bad:
                    assert bool((out[i, seen:, :, 3] == bad).all())     # (its weight is not zero)
                    rest = [d for d in range(dim) if d != 3]
                    # added in another order and from weights that are not rounded: each within h (|O| + sum p |v|)
                    a, b = out[i][:, :, rest].float(), clean[i][:, :, rest].float()
                    h = torch.finfo(c.q.dtype).eps / 2
                    assert bool(((a - b).abs() <= 2.1 * h * (b.abs() + c.values[i].float().abs().max())).all())
                elif what is c.v:
                    assert bool(out[i, seen:, :, 3].isnan().all())
                else:
                    # a score of -inf is a weight of zero; one of +inf or NaN makes its row NaN
                    q = c.q[i, seen:, :, 3].float() * bad
                    hot = ~(q == float("-inf"))
                    assert bool(out[i, seen:][hot].isnan().all())
                    assert bool(out[i, seen:][~hot].isfinite().all())
                assert torch.equal(out[i, :seen], clean[i, :seen])
                others = [j for j in range(4) if j != i]
                assert torch.equal(out[others], clean[others])
                what[page, row] = keep


def test_scores_of_minus_infinity_alone_are_not_no_states():
    for cols in (None, 3000):
        c = Cache([40, 40], 2, 4, 2, 64, "bf16", 16, cols=cols)
        c.q[0, 0, 0] = float("-inf")
        c.q[0, 0, 0, 1:] = 0.0
        page, row = c.at(0, 0, 40)
        c.k[page, row, 0, 0] = 1.0
        out, lse = torch.empty_like(c.q), torch.empty(2, 4, 2, device="cuda")
        run(c, out, lse)
        assert bool(out[0, 0, 0].isnan().all()) and bool(lse[0, 0, 0].isnan())
        assert bool(out[0, 1].isfinite().all()) and bool(out[1].isfinite().all()) and bool(out[0, 0, 1:].isfinite().all())


@pytest.mark.parametrize("scale", [0.0, 1e-3, 2.0])
def test_scales(scale):
    check(Cache([77, 300, 0], 3, 4, 2, 64, "fp16", 16), scale=scale)


def test_no_lse():
    check(Cache([77, 300, 0], 1, 4, 2, 64, "fp16", 16), lse=False)


STRIDE = 1 << 23                                       # 300 pages of it: the last lies 2.5e9 elements into its buffer


@pytest.mark.parametrize("group", [4, 20])
@pytest.mark.parametrize("cols", [150, 3000])
def test_more_than_32_bits_of_offset(cols, group):
    c = Cache([900, 1500, 2300], 2, 2 * group, 2, 64, "bf16", 16, cols=cols, spare=5)
    near = torch.empty_like(c.q)
    run(c, near)
    pages = c.k.shape[0]
    assert pages * STRIDE > 1 << 31
    buf = torch.empty(pages * STRIDE, dtype=torch.bfloat16, device="cuda")
    far = [torch.as_strided(buf, c.k.shape, (STRIDE, *c.k.stride()[1:]), at) for at in (0, 1 << 20)]
    for f, t in zip(far, (c.k, c.v)):
        f.copy_(t)
    c.k, c.v = far
    out = torch.empty_like(c.q)
    run(c, out)
    assert torch.equal(out, near)
    # appending there
    new = torch.randn(3, 2, 2, 64, device="cuda").bfloat16()
    append(c, new, new + 1)
    for i in range(3):
        page, row = c.at(i, c.lens_host[i] - 2, 2)
        assert torch.equal(c.k[page, row], new[i]) and torch.equal(c.v[page, row], new[i] + 1)


def append(c, k_new, v_new, stream=None):
    B.cache_append(c.shape(torch.empty_like(c.q), None, k_new, v_new), k_new, v_new, c.k, c.v, c.table, c.lens, c.slot_of,
                   c.new_lens, stream or torch.cuda.current_stream())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout,page_rows", [("rows", 16), ("heads", 5), ("joint", 64), ("padded", 1)])
@pytest.mark.parametrize("rows,hk,dim", [(1, 8, 128), (7, 3, 40), (130, 1, 8)])
def test_append(dtype, layout, page_rows, rows, hk, dim):
    lens = [rows + 20, rows, max(rows - 1, 0), 0, rows + 400, 300]
    news = [rows, rows, rows, rows, rows // 2, -1]
    c = Cache(lens, rows, 2 * hk, hk, dim, dtype, page_rows, layout, slots=[2, 0, 1, 4, -7, 3], news=news, poison=False)
    # the new tokens' projections lie side by side
    qkv = torch.randn(len(lens), rows, 4 * hk, dim, device="cuda").to(c.q.dtype)
    k_new, v_new = qkv[:, :, 2 * hk:3 * hk], qkv[:, :, 3 * hk:]
    want = [p.clone() for p in c.pools]
    views = dict(zip(("k", "v"), (c.k, c.v)))
    got = [p.clone() for p in c.pools]
    for i, n in c.there():
        for t in range(n):
            pos = lens[i] - n + t
            if pos >= 0:
                page, row = c.at(i, pos, 1)
                views["k"][page, row] = k_new[i, t]
                views["v"][page, row] = v_new[i, t]
    want = [p.clone() for p in c.pools]
    for p, g in zip(c.pools, got):
        p.copy_(g)
    append(c, k_new, v_new)
    for p, w in zip(c.pools, want):
        assert torch.equal(p, w)


def test_append_passes_over_pages_that_are_not_there():
    c = Cache([33, 20], 20, 2, 2, 64, "bf16", 16, poison=False)
    before = [p.clone() for p in c.pools]
    ids = c.table.clone()
    c.table[0, 1], c.table[1, 1] = -4, c.k.shape[0]
    new = torch.randn(2, 20, 2, 64, device="cuda").bfloat16()
    append(c, new, new)
    for p, b in zip((c.k, c.v), before):
        for w in (ids[0, 1], ids[1, 1]):
            assert torch.equal(p[w], b[w])
        assert torch.equal(p[ids[0, 0], 13:], new[0, :3]) and torch.equal(p[ids[0, 2], :1], new[0, 19:])
        assert torch.equal(p[ids[1, 0]], new[1, :16])


def test_empty_sizes():
    c = Cache([33, 20], 1, 2, 2, 64, "bf16", 16)
    q = c.q
    for cut in (q[:0], q[:, :0]):
        out = torch.empty_like(cut)
        shape = B.PagedShape.of(cut, c.k, c.v, out, c.table)
        B.paged_attn(shape, cut, c.k, c.v, c.table, c.lens, None, None, out, None, None, 0)
    out, lse = torch.full_like(q, 7), torch.full((2, 2, 1), 7.0, device="cuda")
    shape = B.PagedShape.of(q, c.k[:0], c.v[:0], out, c.table)
    n = B.paged_attn_scratch_bytes(shape)
    scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    B.paged_attn(shape, q, None, None, None, c.lens, None, None, out, lse, scratch, n, torch.cuda.current_stream())
    assert not out.any() and bool((lse == float("-inf")).all())
    out.fill_(7)
    shape = B.PagedShape.of(q, c.k, c.v, out, c.table[:0])
    B.paged_attn(shape, q, c.k, c.v, c.table, None, None, None, out, None, None, 0)
    assert bool((out == 7).all())


@pytest.mark.parametrize("cols", [40, 3000])
def test_captured_while_sequences_grow(cols):
    """One graph of append and attention, replayed as the lengths on the device change."""
    c = Cache([16, 100, 33], 1, 8, 2, 64, "bf16", 16, cols=cols, spare=60)
    free = [p for p in range(c.k.shape[0]) if p not in set(c.table[c.table >= 0].tolist())]
    for i in range(3):                                 # pages for what is to come
        have = cdiv(c.lens_host[i], 16)
        c.table[i, have:have + 4] = torch.tensor([free.pop() for _ in range(4)], dtype=torch.int32)
    new = torch.empty(2, 3, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(c.q), torch.empty(3, 8, 1, device="cuda")
    shape = c.shape(out, None, new[0], new[1])
    n = B.paged_attn_scratch_bytes(shape)
    scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream()
        B.cache_append(shape, new[0], new[1], c.k, c.v, c.table, c.lens, None, None, s)
        B.paged_attn(shape, c.q, c.k, c.v, c.table, c.lens, None, None, out, lse, scratch, n, s)
    for step in range(40):
        c.lens += 1
        new.normal_()
        c.q.normal_()
        for i in range(3):
            c.lens_host[i] += 1
            c.keys[i], c.values[i] = torch.cat([c.keys[i], new[0, i]]), torch.cat([c.values[i], new[1, i]])
        graph.replay()
        if step % 13 == 0 or step == 39:
            got = out.clone(), lse.clone()
            want = check(c)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_calls_overlap_on_two_streams():
    caches = [Cache([900, 1500, 20], 1, 8, 2, 128, "bf16", 16, cols=4000, seed=1), Cache([3000] * 40, 2, 8, 4, 64, "fp16", 64, seed=2)]
    sides, want, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    for c in caches:
        out = torch.empty_like(c.q)
        run(c, out)
        want.append(out)
        outs.append(torch.empty_like(out))
    scr = [torch.full((B.paged_attn_scratch_bytes(c.shape(o)) + 64,), 0xFF, dtype=torch.uint8, device="cuda") for c, o in zip(caches, outs)]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, o, side, s in zip(caches, outs, sides, scr):
            with torch.cuda.stream(side):
                run(c, o, stream=side, scratch=s)
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dim", [64, 128])
def test_waits_that_run_out(dim):
    """Nothing is loaded, or the limit is far too short: the call ends, the status says so, the next one is right."""
    c = Cache([3000, 700], 4, 32, 2, dim, "bf16", 16, cols=4000)
    want, out = torch.empty_like(c.q), torch.empty_like(c.q)
    run(c, want)
    stream = torch.cuda.current_stream()
    scratch = torch.full((B.paged_attn_scratch_bytes(c.shape(out)) + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    try:
        B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 1_000_000)
        B.debug_set(B.DEBUG_SKIP_NEXT_XATTN_LOADS, 1)
        run(c, out, stream=stream, scratch=scratch)
        assert B.device_status(stream)[0] == B.ERR_DEVICE_TIMEOUT
        B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 1)
        for _ in range(20):
            run(c, out, stream=stream, scratch=scratch)
            assert B.device_status(stream)[0] in (B.OK, B.ERR_DEVICE_TIMEOUT)
    finally:
        B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 0)
    run(c, out)
    assert torch.equal(out, want)


def test_strides_of_sizes_of_one_do_not_matter():
    c = Cache([50], 1, 1, 1, 64, "bf16", 64)
    out = torch.empty_like(c.q)
    shape = c.shape(out)
    for f in ("q_stride", "o_stride"):
        setattr(shape, f, (ctypes.c_int64 * 3)(3, 0, -5))
    shape.table_stride = 0
    shape.k_stride[2], shape.v_stride[2] = 1, 0
    n = B.paged_attn_scratch_bytes(shape)
    scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    B.paged_attn(shape, c.q.data_ptr(), c.k.data_ptr(), c.v.data_ptr(), c.table.data_ptr(), c.lens, None, None, out.data_ptr(), None,
                 scratch, n, torch.cuda.current_stream())
    want = torch.empty_like(c.q)
    run(c, want)
    assert torch.equal(out, want)
