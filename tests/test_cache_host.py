"""CPU-only checks of the paged cache's operators: bad arguments are refused before any CUDA call, scratch sizes, and what the
binding refuses of the tensors themselves."""
import ctypes

import pytest
import torch

from paper_2506_09092_b200 import binding as B
from paper_2506_09092_b200 import build as libbuild

P = 1 << 20             # a non-null, aligned stand-in address; never dereferenced on error
I3 = ctypes.c_int64 * 3
STRIDES = ("q_stride", "o_stride", "kn_stride", "vn_stride", "k_stride", "v_stride")


@pytest.fixture(scope="module", autouse=True)
def built():
    libbuild.build()


def shape(**k):
    a = dict(batch=3, q_rows=2, q_heads=8, kv_heads=4, head_dim=64, pages=50, page_rows=16, slots=5, table_cols=10,
             table_stride=12, q_stride=(1024, 512, 64), o_stride=(1024, 512, 64), kn_stride=(512, 256, 64),
             vn_stride=(512, 256, 64), k_stride=(4096, 256, 64), v_stride=(4096, 256, 64), dtype=B.BF16, scale=0.125)
    a.update(k)
    for f in STRIDES:
        a[f] = I3(*a[f])
    return B.PagedShape(**a)


def attn(s, **k):
    a = dict(q=P, k=P, v=P, table=P, lens=P, slot_of=P, new_lens=P, o=P, lse=P, scratch=P, scratch_bytes=1 << 40)
    a.update(k)
    return B.paged_attn(s, check=False, **a)


def append(s, **k):
    a = dict(k_new=P, v_new=P, k=P, v=P, table=P, lens=P, slot_of=P, new_lens=P)
    a.update(k)
    return B.cache_append(s, check=False, **a)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=B.F32), B.ERR_INVALID_DTYPE), (dict(dtype=7), B.ERR_INVALID_DTYPE),
    *[(dict([(f, -1)]), B.ERR_INVALID_DIM) for f in ("batch", "q_rows", "q_heads", "kv_heads", "head_dim", "pages", "slots", "table_cols")],
    *[(dict([(f, 1 << 31)]), B.ERR_INVALID_DIM) for f in ("batch", "q_rows", "pages", "page_rows", "slots", "table_cols")],
    (dict(page_rows=0), B.ERR_INVALID_DIM), (dict(kv_heads=3), B.ERR_INVALID_DIM), (dict(kv_heads=0), B.ERR_INVALID_DIM),
    (dict(table_cols=1 << 20, table_stride=1 << 20, page_rows=1 << 11), B.ERR_INVALID_DIM),
    (dict(batch=1 << 20, q_rows=1 << 10), B.ERR_INVALID_DIM),
    (dict(scale=-1.0), B.ERR_INVALID_DIM), (dict(scale=float("nan")), B.ERR_INVALID_DIM), (dict(scale=float("inf")), B.ERR_INVALID_DIM),
    (dict(table_stride=9), B.ERR_INVALID_LD), (dict(table_stride=1 << 50), B.ERR_INVALID_DIM),
    (dict(head_dim=60), B.ERR_UNSUPPORTED_SHAPE), (dict(head_dim=136), B.ERR_UNSUPPORTED_SHAPE),
    (dict(k_stride=(4096, 256, 56)), B.ERR_INVALID_LD), (dict(v_stride=(4088, 256, 64)), B.ERR_INVALID_LD),
    (dict(v_stride=(4096, -256, 64)), B.ERR_INVALID_LD), (dict(k_stride=(4100, 256, 64)), B.ERR_UNSUPPORTED_SHAPE),
    (dict(k_stride=(1 << 45, 256, 64)), B.ERR_INVALID_DIM),
])
def test_shape_refusals(change, status):
    s = shape(**change)
    assert attn(s) == append(s) == status
    assert B.paged_attn_scratch_bytes(s) == 0


def test_operand_refusals():
    s = shape()
    for name in ("q", "k", "v", "o"):
        assert attn(s, **{name: None}) == B.ERR_INVALID_POINTER
        assert attn(s, **{name: P + 8}) == B.ERR_UNSUPPORTED_SHAPE
    for name in ("k_new", "v_new", "k", "v"):
        assert append(s, **{name: None}) == B.ERR_INVALID_POINTER
        assert append(s, **{name: P + 8}) == B.ERR_UNSUPPORTED_SHAPE
    for name in ("table", "lens"):
        assert attn(s, **{name: None}) == append(s, **{name: None}) == B.ERR_INVALID_POINTER
    for name in ("table", "lens", "slot_of", "new_lens"):
        assert attn(s, **{name: P + 2}) == append(s, **{name: P + 2}) == B.ERR_MISALIGNED
    assert attn(s, lse=P + 2) == B.ERR_MISALIGNED
    assert attn(shape(q_stride=(1024, 512, 56))) == attn(shape(o_stride=(512, 512, 64))) == B.ERR_INVALID_LD
    assert append(shape(kn_stride=(512, 256, 8))) == append(shape(vn_stride=(256, 256, 64))) == B.ERR_INVALID_LD
    # what a call does not use is not looked at
    big = shape(batch=200, kv_heads=8, k_stride=(8192, 512, 64), v_stride=(8192, 512, 64), kn_stride=(-1, 0, 0))
    need = B.paged_attn_scratch_bytes(big)
    assert need > 0
    for scratch, size in ((None, need), (P + 8, need), (P, need - 1)):
        assert attn(big, scratch=scratch, scratch_bytes=size) == B.ERR_WORKSPACE
    assert B.lib().cudallm_paged_attn(None, *[P] * 10, 1 << 30, None) == B.ERR_INVALID_POINTER
    assert B.lib().cudallm_cache_append(None, *[P] * 8, None) == B.ERR_INVALID_POINTER


def test_empty_sizes():
    for change in (dict(batch=0), dict(q_rows=0), dict(head_dim=0), dict(slots=0), dict(q_heads=0, kv_heads=0)):
        s = shape(**change)
        assert attn(s, q=None, k=None, v=None, o=None, table=None, lens=None) == B.OK
        assert append(s, k_new=None, v_new=None, k=None, v=None, table=None, lens=None) == B.OK
        assert B.paged_attn_scratch_bytes(s) == 0
    for change in (dict(pages=0), dict(table_cols=0)):
        assert append(shape(**change), k_new=None, v_new=None, k=None, v=None, table=None, lens=None) == B.OK


def test_pool_refusals():
    def copy(pools=((P, 64, 64),), pages=4, src=P, dst=P, n=2, count=None):
        array = (B.CPagePool * max(len(pools), 1))()
        for e, (data, stride, size) in zip(array, pools):
            e.data, e.stride, e.bytes = data, stride, size
        return B.lib().cudallm_pages_copy(array, len(pools) if count is None else count, pages, src, dst, n, None)
    assert copy(count=-1) == copy(count=65537) == copy(pages=-1) == copy(n=-1) == copy(n=1 << 31) == copy(pages=1 << 31) == B.ERR_INVALID_DIM
    assert copy([(P, 64, -16)]) == copy([(P, 1 << 45, 64)], 1 << 10) == copy([(P, 64, 1 << 47)]) == B.ERR_INVALID_DIM
    assert copy([(None, 64, 64)]) == copy(src=None) == copy(dst=None) == B.ERR_INVALID_POINTER
    assert copy([(P, 48, 64)]) == B.ERR_INVALID_LD
    assert copy([(P + 8, 64, 64)]) == copy([(P, 72, 64)]) == copy([(P, 64, 56)]) == B.ERR_UNSUPPORTED_SHAPE
    assert copy(src=P + 2) == copy(dst=P + 1) == B.ERR_MISALIGNED
    assert copy(n=0, src=None) == copy([]) == copy(pages=0) == B.OK
    assert B.lib().cudallm_pages_copy(None, 1, 4, P, P, 1, None) == B.ERR_INVALID_POINTER


def c_book(**k):
    a = dict(refs=P, lens=P, table=P, pages=100, page_rows=8, slots=6, table_cols=9, table_stride=9)
    a.update(k)

    class Book:
        c = B.CPageBook(**a)

        def _here(self):
            return self.c
    return Book()


def book_calls(book, n=4, **k):
    a = dict(scratch=P, scratch_bytes=1 << 40)
    a.update(k)
    return (B.pages_fork(book, P, P, n, check=False, **a), B.pages_resize(book, None, P, P, n, P, check=False, **a),
            B.pages_compact(book, None, P, check=False, **a))


@pytest.mark.parametrize("change,status", [
    (dict(refs=None), B.ERR_INVALID_POINTER), (dict(lens=None), B.ERR_INVALID_POINTER), (dict(table=None), B.ERR_INVALID_POINTER),
    (dict(refs=P + 4), B.ERR_MISALIGNED), (dict(lens=P + 2), B.ERR_MISALIGNED),
    (dict(table=P + 2), B.ERR_MISALIGNED),
    (dict(pages=-1), B.ERR_INVALID_DIM), (dict(pages=(1 << 20) + 1), B.ERR_INVALID_DIM), (dict(page_rows=0), B.ERR_INVALID_DIM),
    (dict(slots=-1), B.ERR_INVALID_DIM), (dict(table_cols=-1), B.ERR_INVALID_DIM),
    (dict(table_cols=1 << 28, table_stride=1 << 28), B.ERR_INVALID_DIM),
    (dict(table_stride=8), B.ERR_INVALID_LD), (dict(table_stride=1 << 50), B.ERR_INVALID_DIM),
])
def test_book_refusals(change, status):
    book = c_book(**change)
    assert set(book_calls(book)) == {status}
    assert B.pages_fork_scratch_bytes(book, 4) == B.pages_resize_scratch_bytes(book, 4) == B.pages_compact_scratch_bytes(book) == 0


def test_book_call_refusals():
    book = c_book()
    assert book_calls(book, n=-1)[:2] == book_calls(book, n=16385)[:2] == (B.ERR_INVALID_DIM,) * 2
    for k in (dict(scratch=None), dict(scratch=P + 8), dict(scratch_bytes=15)):
        assert set(book_calls(book, **k)) == {B.ERR_WORKSPACE}
    assert B.pages_fork(book, None, P, 1, P, 1 << 30, check=False) == B.pages_fork(book, P, None, 1, P, 1 << 30, check=False) == B.ERR_INVALID_POINTER
    assert B.pages_fork(book, P + 2, P, 1, P, 1 << 30, check=False) == B.ERR_MISALIGNED
    assert B.pages_fork(book, None, None, 0, None, 0, check=False) == B.OK
    resize = lambda slots=P, lens=P, n=3, result=P: B.pages_resize(book, None, slots, lens, n, result, P, 1 << 30, check=False)
    assert resize(lens=None) == B.ERR_INVALID_POINTER and resize(slots=None, n=7) == B.ERR_INVALID_DIM
    assert resize(slots=P + 2) == resize(lens=P + 2) == resize(result=P + 2) == B.ERR_MISALIGNED
    assert B.pages_compact(book, None, P + 1, P, 1 << 30, check=False) == B.ERR_MISALIGNED
    bad = (B.CPagePool * 1)(B.CPagePool(P, 64, 72))
    assert B.lib().cudallm_pages_resize(book.c, bad, 1, P, P, 1, P, P, 1 << 30, None) == B.ERR_INVALID_LD
    assert B.lib().cudallm_pages_compact(book.c, bad, 1, P, P, 1 << 30, None) == B.ERR_INVALID_LD
    assert B.lib().cudallm_pages_compact(None, None, 0, P, P, 1 << 30, None) == B.ERR_INVALID_POINTER


def verify(**k):
    a = dict(p=P, q=P, drafts=P, draft_lens=P, u=P, tokens=P, accepted=P, batch=3, n=2, vocab=100, ldp=100, ldq=100, dtype=B.F32)
    a.update(k)
    return B.draft_verify(**a, check=False)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), B.ERR_INVALID_DTYPE), (dict(dtype=-1), B.ERR_INVALID_DTYPE),
    (dict(batch=-1), B.ERR_INVALID_DIM), (dict(n=-1), B.ERR_INVALID_DIM), (dict(vocab=0), B.ERR_INVALID_DIM),
    (dict(vocab=1 << 31, ldp=1 << 31, ldq=1 << 31), B.ERR_INVALID_DIM), (dict(batch=1 << 30), B.ERR_INVALID_DIM),
    (dict(n=1 << 31), B.ERR_INVALID_DIM), (dict(ldp=1 << 44), B.ERR_INVALID_DIM), (dict(ldq=1 << 44), B.ERR_INVALID_DIM),
    (dict(ldp=99), B.ERR_INVALID_LD), (dict(ldq=99), B.ERR_INVALID_LD),
    (dict(p=None), B.ERR_INVALID_POINTER), (dict(drafts=None), B.ERR_INVALID_POINTER), (dict(u=None), B.ERR_INVALID_POINTER),
    (dict(tokens=None), B.ERR_INVALID_POINTER), (dict(accepted=None), B.ERR_INVALID_POINTER),
    (dict(p=P + 2), B.ERR_MISALIGNED), (dict(q=P + 2), B.ERR_MISALIGNED), (dict(p=P + 1, dtype=B.BF16), B.ERR_MISALIGNED),
    *[(dict([(f, P + 2)]), B.ERR_MISALIGNED) for f in ("drafts", "draft_lens", "u", "tokens", "accepted")],
    (dict(batch=0, p=None, u=None), B.OK),
])
def test_verify_refusals(change, status):
    assert verify(**change) == status


def test_struct_layouts():
    assert ctypes.sizeof(B.PagedShape) == 232 and ctypes.sizeof(B.CPagePool) == 24 and ctypes.sizeof(B.CPageBook) == 64


# ------------------------------------------------------------- the binding --
def operands(t=torch.bfloat16):
    q = torch.zeros(3, 2, 8, 64, dtype=t)
    pool = torch.zeros(50, 2, 16, 4, 64, dtype=t)
    new = torch.zeros(3, 2, 2, 4, 64, dtype=t)
    table, lens = torch.zeros(5, 10, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    return dict(q=q, k=pool[:, 0], v=pool[:, 1], k_new=new[:, :, 0], v_new=new[:, :, 1], table=table, lens=lens, slot_of=torch.zeros(3, dtype=torch.int32),
                new_lens=torch.zeros(3, dtype=torch.int32), o=torch.zeros_like(q), lse=torch.zeros(3, 8, 2))


def shape_of(a):
    return B.PagedShape.of(a["q"], a["k"], a["v"], a["o"], a["table"], a["k_new"], a["v_new"])


def call_attn(s, a):
    B.paged_attn(s, a["q"], a["k"], a["v"], a["table"], a["lens"], a["slot_of"], a["new_lens"], a["o"], a["lse"], None, 0)


def call_append(s, a):
    B.cache_append(s, a["k_new"], a["v_new"], a["k"], a["v"], a["table"], a["lens"], a["slot_of"], a["new_lens"])


def test_shape_from_tensors():
    a = operands()
    s = shape_of(a)
    assert (s.batch, s.q_rows, s.q_heads, s.kv_heads, s.head_dim, s.pages, s.page_rows, s.slots, s.table_cols) == (3, 2, 8, 4, 64, 50, 16, 5, 10)
    assert list(s.k_stride) == [2 * 16 * 256, 256, 64] and list(s.kn_stride) == [2 * 512, 512, 64] and s.scale == 0.125
    for name, other in (("q", a["q"].half()), ("v", a["v"].float()), ("v_new", a["v_new"].half())):
        with pytest.raises(TypeError):
            shape_of(dict(a, **{name: other}))
    with pytest.raises(TypeError):
        shape_of({n: t.float() if t.dtype == torch.bfloat16 else t for n, t in a.items()})
    for name, other in (("q", a["q"][0]), ("v", a["v"][:, :8]), ("o", a["o"][:2]), ("k_new", a["k_new"][:, :1]), ("table", a["table"][0]),
                        ("k", a["k"].transpose(2, 3)), ("table", a["table"].t())):
        with pytest.raises(ValueError):
            shape_of(dict(a, **{name: other}))


def test_tensors_as_the_shape_says():
    a = operands()
    s = shape_of(a)
    for call in (call_attn, call_append):
        with pytest.raises(TypeError, match="host memory"):
            call(s, a)
        with pytest.raises(TypeError, match="host memory"):
            call(s, dict(a, slot_of=None, new_lens=None, lse=None))
    for name in ("q", "k", "v", "o", "k_new", "v_new"):
        turned = a[name].transpose(1, 2).contiguous().transpose(1, 2)
        for call, used in ((call_attn, ("q", "k", "v", "o")), (call_append, ("k", "v", "k_new", "v_new"))):
            if name not in used:
                continue
            for other, error in ((a[name].half(), TypeError), (turned, ValueError), (a[name][:-1], ValueError), (torch.zeros(9, dtype=torch.bfloat16), ValueError)):
                with pytest.raises(error, match=f"^{name}"):
                    call(s, dict(a, **{name: other}))
    for name, bad in (("table", a["table"].long()), ("lens", a["lens"].long()), ("slot_of", a["slot_of"].float()), ("new_lens", a["new_lens"].long())):
        for call in (call_attn, call_append):
            with pytest.raises(TypeError, match=f"^{name}"):
                call(s, dict(a, **{name: bad}))
            with pytest.raises(ValueError, match=f"^{name}"):
                call(s, dict(a, **{name: a[name][:2]}))
    for bad, error in ((a["lse"].double(), TypeError), (a["lse"][:2], ValueError)):
        with pytest.raises(error, match="^lse"):
            call_attn(s, dict(a, lse=bad))


def test_pools_and_books_of_tensors(monkeypatch):
    monkeypatch.setattr(B, "_d", lambda *xs: [None if x is None else x if isinstance(x, int) else x.data_ptr() for x in xs])
    pool = torch.zeros(50, 2, 16, 4, 64, dtype=torch.bfloat16)
    both = B.page_pools([pool[:, 0], pool[:, 1]])
    assert both.count == 2 and both.pages == 50 and both.array[0].bytes == 8192 and both.array[1].stride == 16384
    assert B.page_pools([pool]).array[0].bytes == 16384 and B.page_pools([]).count == 0
    for bad in ([pool, pool[:49]], [pool[:, :, 0]], [pool[:, 0].transpose(1, 2)], [pool, pool[:, 1]], [pool[:, 0], pool[:, 0]], [torch.zeros(4)]):
        with pytest.raises(ValueError):
            B.page_pools(bad)
    book = B.PageBook(7, 4, 3, 5, device="cpu")
    assert book.refs.shape == (7,) and book.lens.shape == (3,) and book.table.shape == (3, 5) and not book.data.any()
    assert (book.c.lens - book.c.refs, book.c.table - book.c.refs, book.c.refs) == (32, 48, book.data.data_ptr())
    with pytest.raises(ValueError, match="pools of 50 pages"):
        B.pages_resize(book, both, None, P, 1, None, P, 1 << 20)
    for name, k in (("src", dict(src=torch.zeros(2))), ("dst", dict(dst=torch.zeros(1, dtype=torch.int32)))):
        a = dict(src=P, dst=P)
        a.update(k)
        with pytest.raises((TypeError, ValueError), match=f"^{name}"):
            B.pages_fork(book, a["src"], a["dst"], 2, P, 1 << 20)
        with pytest.raises((TypeError, ValueError), match=f"^{name}"):
            B.pages_copy(both, a["src"], a["dst"], 2)


def test_probabilities_and_vectors_of_verify():
    t = dict(p=torch.zeros(3, 3, 100), q=torch.zeros(3, 2, 100), drafts=torch.zeros(3, 2, dtype=torch.int32),
             draft_lens=torch.zeros(3, dtype=torch.int32), u=torch.zeros(3, 3), tokens=torch.zeros(3, 3, dtype=torch.int32),
             accepted=torch.zeros(3, dtype=torch.int32))
    call = lambda **k: B.draft_verify(**dict(t, batch=3, n=2, vocab=100, ldp=100, ldq=100, dtype=B.F32, **k))
    with pytest.raises(TypeError, match="host memory"):
        call()
    for name, bad, error in (("p", t["p"].half(), TypeError), ("q", t["q"].double(), TypeError), ("p", t["p"][:2], ValueError),
                             ("q", t["q"][:, :, :99], ValueError), ("p", t["p"].transpose(1, 2), ValueError),
                             ("drafts", t["drafts"].long(), TypeError), ("u", t["u"].double(), TypeError), ("u", t["u"][:2], ValueError),
                             ("tokens", t["tokens"][:, :2], ValueError), ("accepted", t["accepted"][:1], ValueError),
                             ("draft_lens", t["draft_lens"].long(), TypeError)):
        with pytest.raises(error, match=f"^{name}"):
            B.draft_verify(**dict(dict(t, batch=3, n=2, vocab=100, ldp=100, ldq=100, dtype=B.F32), **{name: bad}))
