"""CPU-only checks of the paged cache's operators, beside test_cache_host.py: scales at their ends, and tensors that
are not laid out as a call reads them."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B
from paper_2506_09092_b200 import build as libbuild
from test_cache_host import P, append, attn, shape


@pytest.fixture(scope="module", autouse=True)
def built():
    libbuild.build()


def test_a_scale_whose_product_is_no_number_is_refused():
    s = shape(scale=2.4e38)                            # log2 e times as much is above 3.4e38
    assert attn(s) == append(s) == B.ERR_INVALID_DIM and B.paged_attn_scratch_bytes(s) == 0
    for scale in (0.0, 1e-45, 2.0e38):
        assert attn(shape(scale=scale), q=None) == B.ERR_INVALID_POINTER


# ------------------------------------------------------------- the binding --
class _Nothing:
    """In the library's place: takes every call, reads nothing."""

    def __getattr__(self, name):
        return lambda *a: B.OK


@pytest.fixture
def addresses(monkeypatch):
    """Tensors in host memory pass for the device's, and no call is made."""
    monkeypatch.setattr(B, "_d", lambda *xs: [None if x is None else x if isinstance(x, int) else x.data_ptr() for x in xs])
    monkeypatch.setattr(B, "lib", lambda: _Nothing())


def verify(batch=3, n=2, vocab=100, ldp=None, ldq=None, **k):
    a = dict(p=torch.zeros(batch, n + 1, vocab), q=torch.zeros(batch, n, vocab), drafts=torch.zeros(batch, n, dtype=torch.int32),
             draft_lens=None, u=torch.zeros(batch, n + 1), tokens=torch.zeros(batch, n + 1, dtype=torch.int32),
             accepted=torch.zeros(batch, dtype=torch.int32))
    a.update(k)
    return B.draft_verify(**a, batch=batch, n=n, vocab=vocab, ldp=ldp or vocab, ldq=ldq or vocab, dtype=B.F32)


def test_rows_of_probabilities_lie_at_the_pitch(addresses):
    big, wide = torch.zeros(3, 6, 100), torch.zeros(3, 3, 128)
    for name, per in (("p", 3), ("q", 2)):
        for bad, ld in ((big[:, :per], 100), (big[:, 1:1 + per], 100), (big, 100), (big[:, ::2], 100), (big[:, :per], 200), (wide, 100),
                        (wide[:, :per, :100], 100), (wide.view(9, 128), 100), (wide.view(9, 128)[:, :100], 100),
                        (torch.zeros(6, 3, 100).transpose(0, 1), 100), (big[:, :1].expand(3, 6, 100), 100),
                        (torch.zeros(3, 12, 50)[:, :2 * per], 100)):
            with pytest.raises(ValueError, match=f"^{name}"):
                verify(**{name: bad, "ld" + name: ld})


def test_rows_that_lie_at_the_pitch_are_taken_however_the_tensor_is_shaped(addresses):
    wide = torch.zeros(3, 3, 128)
    for good, ld in ((torch.zeros(9, 100), 100), (torch.zeros(1, 9, 100), 100), (torch.zeros(9, 1, 100), 100), (torch.zeros(900), 100), (torch.zeros(5000), 100),
                     (torch.zeros(20, 100), 100), (torch.zeros(3, 300), 100), (torch.zeros(3, 3, 4, 25), 100), (wide, 128),
                     (wide[:, :, :100], 128), (wide[:, :, 28:], 128), (wide.view(9, 128)[:, :100], 128), (torch.zeros(18, 100)[::2], 200),
                     (torch.zeros(1200)[30:], 100)):
        assert verify(p=good, ldp=ld) == B.OK
    assert verify(batch=1, n=0, q=None, p=torch.zeros(1, 4, 100)[:, 2:3]) == B.OK
    assert verify(batch=1, p=torch.zeros(1, 7, 100), q=torch.zeros(2, 5, 100)[1:, :2]) == B.OK
    assert verify(batch=4, n=1, p=torch.zeros(4, 2, 100), q=torch.zeros(4, 2, 100)[:, 1:], ldq=200) == B.OK
    assert verify(batch=2, n=3, vocab=1, p=torch.zeros(2, 4, 1), q=torch.zeros(2, 3, 1)) == B.OK


def test_vectors_with_more_than_a_sequence_has(addresses):
    for name, bad in (("drafts", torch.zeros(3, 5, dtype=torch.int32)), ("u", torch.zeros(3, 4)), ("tokens", torch.zeros(3, 9, dtype=torch.int32))):
        with pytest.raises(ValueError, match=f"^{name}"):
            verify(**{name: bad})
    assert verify(u=torch.zeros(50), drafts=torch.zeros(7, dtype=torch.int32), tokens=torch.zeros(2, 9, dtype=torch.int32)) == B.OK


class _OnDevice(torch.Tensor):
    """A host tensor that says it is on a device."""
    device_index = 0

    def get_device(self):
        return self.device_index


def on(index, *size, dtype=torch.bfloat16):
    t = torch.zeros(*size, dtype=dtype).as_subclass(_OnDevice)
    t.device_index = index
    return t


def test_pools_of_another_device_than_the_current_one(monkeypatch):
    """A table of pools was built under one device and a call is made under another: its addresses mean nothing there."""
    monkeypatch.setattr(B, "lib", lambda: _Nothing())
    monkeypatch.setattr(B, "_get_device", lambda: 0)
    pools = B.page_pools([on(0, 50, 64), on(0, 50, 64)])
    with pytest.raises(ValueError, match="device 1, the current device is 0"):
        B.page_pools([on(1, 50, 64)])
    with pytest.raises(ValueError, match="device 1, the current device is 0"):
        B.page_pools([on(0, 50, 64), on(1, 50, 64)])
    assert B.pages_copy(pools, P, P, 2) == B.OK
    book, scratch = B.PageBook(50, 4, 3, 5, device="cpu"), 1 << 20
    book.data = on(0, 80, dtype=torch.int32)
    calls = (lambda: B.pages_resize(book, pools, None, P, 1, None, P, scratch), lambda: B.pages_compact(book, pools, None, P, scratch))
    assert all(c() == B.OK for c in calls)
    monkeypatch.setattr(B, "_get_device", lambda: 1)
    book.data = on(1, 80, dtype=torch.int32)
    for call in (lambda: B.pages_copy(pools, P, P, 2), *calls):
        with pytest.raises(ValueError, match="device 0, the current device is 1"):
            call()
    assert B.pages_resize(book, None, None, P, 1, None, P, scratch) == B.OK
    assert B.pages_copy(B.page_pools([]), P, P, 2) == B.OK
