"""CPU-only: overlaps that the table of gradients refuses and those that it takes.  Every CTA scales its own piece at its
own time, so what one entry writes no other entry may read."""
import itertools

import pytest
import torch

from paper_2506_09092_b200 import binding as B


@pytest.fixture(autouse=True)
def host_addresses(monkeypatch):
    """Host tensors stand in for device ones: the table only looks at addresses."""
    monkeypatch.setattr(B, "_d", lambda *xs: [x.data_ptr() for x in xs])


def refused(tensors, outs=None):
    try:
        B.tensor_table(tensors, outs)
    except ValueError:
        return True
    return False


def test_in_place_over_what_another_entry_reads():
    t, u, w = torch.zeros(100), torch.zeros(100), torch.zeros(100)
    assert refused([t, t], [t, u]) and refused([t, t], [u, t])
    assert refused([t, t[50:]], [t, u[50:]]) and refused([t[50:], t], [u[50:], t])
    assert refused([t[:60], t[40:]], [t[:60], u[:60]]) and refused([t[:60], t[40:]], [u[:60], t[40:]])
    assert refused([w, t[:60], u, t[59:60]], [w, t[:60], u, w.new_zeros(1)])
    assert not refused([t[:50], t[50:]], [t[:50], u[:50]]) and not refused([t, t], [u, w])
    assert not refused([t, u], [t, w]) and not refused([t[:0], t], [t[:0], u]) and not refused([t, t[:0]], [t, u[:0]])


def test_every_pair_of_ranges():
    """Two entries over a buffer of six elements, inputs and outputs anywhere: refused if and only if an
    output meets the other output, or an input that is not its own in place."""
    buf = torch.zeros(6)
    spans = [(b, b + n) for n in (2,) for b in range(5)]
    meets = lambda a, b: a[0] < b[1] and b[0] < a[1]
    for i0, o0, i1, o1 in itertools.product(spans, repeat=4):
        outs_in = [(o, i) for (k, o), (m, i) in itertools.product(enumerate((o0, o1)), enumerate((i0, i1))) if not (k == m and o == i)]
        want = meets(o0, o1) or any(meets(o, i) for o, i in outs_in)
        cut = [buf[a:b] for a, b in (i0, i1, o0, o1)]
        assert refused(cut[:2], cut[2:]) == want, (i0, o0, i1, o1)
