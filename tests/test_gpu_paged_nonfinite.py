"""Scores of minus infinity, whichever way the keys are shared out.  (Tolerances as in paged_util.)"""
import pytest
import torch

from paged_util import Cache, check, run

pytestmark = pytest.mark.gpu

FORMS = [(1, 1, 16, None), (1, 4, 16, None), (1, 4, 16, 3000), (4, 4, 7, 3000), (5, 4, 24, None), (5, 8, 24, 3000), (5, 8, 16, 3000),
         (2, 50, 64, 3000)]


def keys_of_minus_infinity(c, i, positions):
    """Every query's product with these keys is -inf: a weight of zero."""
    page, row = c.at(i, 0, c.lens_host[i])
    at = torch.tensor(positions, device="cuda")
    c.k[page[at], row[at], :, 3] = float("-inf")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,group,page_rows,cols", FORMS)
def test_scores_of_minus_infinity_weigh_nothing_wherever_they_lie(rows, group, page_rows, cols, dim):
    """A warp's, a CTA's or a part's share of the keys may hold such scores alone; the others' decide then."""
    lens = [700, 9000, 40, 130, 65]
    c = Cache(lens, rows, 2 * group, 2, dim, "bf16", page_rows, cols=cols, seed=rows + group)
    c.q[..., 3] = c.q[..., 3].abs() + 0.5
    keep = [{5}, {0, 4444}, {33}, set(range(64)), set(range(1, 60))]
    absent = [[s for s in range(n) if s not in k] for n, k in zip(lens, keep)]
    for i, a in enumerate(absent):
        keys_of_minus_infinity(c, i, a)
    check(c, absent=absent)


@pytest.mark.parametrize("rows,group,page_rows,cols", FORMS)
def test_scores_of_minus_infinity_alone_make_no_number(rows, group, page_rows, cols):
    """... however many parts they come in; and tokens without a state stay apart from that."""
    lens = [9000, rows, 300, 0]
    c = Cache(lens, rows, 2 * group, 2, 64, "bf16", page_rows, cols=cols, seed=rows)
    c.q[..., 3] = c.q[..., 3].abs() + 0.5
    clean, out, lse = torch.empty_like(c.q), torch.empty_like(c.q), torch.empty(4, 2 * group, rows, device="cuda")
    run(c, clean)
    keys_of_minus_infinity(c, 0, list(range(9000)))
    run(c, out, lse)
    assert bool(out[0].isnan().all()) and bool(lse[0].isnan().all())
    assert torch.equal(out[1:], clean[1:]) and bool(lse[1:3].isfinite().all())
    assert not out[3].any() and bool((lse[3] == float("-inf")).all())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,group,page_rows,cols", FORMS)
def test_a_value_that_is_not_finite_under_a_weight_of_zero(rows, group, page_rows, cols, dim):
    """0 x inf is NaN, in its own column only, wherever the weight of zero comes from."""
    lens, keep = [700, 9000, 130], [{5}, {0, 4444}, set(range(64))]
    c = Cache(lens, rows, 2 * group, 2, dim, "bf16", page_rows, cols=cols, seed=rows + group)
    c.q[..., 3] = c.q[..., 3].abs() + 0.5
    for i, k in enumerate(keep):
        keys_of_minus_infinity(c, i, [s for s in range(lens[i]) if s not in k])
    clean, out = torch.empty_like(c.q), torch.empty_like(c.q)
    run(c, clean)
    for i, at in ((0, 600), (1, 8000), (2, 130 - rows), (2, 100)):
        page, row = c.at(i, at, 1)
        keep = c.v[page, row].clone()
        c.v[page, row, :, 9] = float("inf")
        run(c, out)
        assert bool(out[i, :, :, 9].isnan().all())
        rest = [d for d in range(dim) if d != 9]
        assert torch.equal(out[i][:, :, rest], clean[i][:, :, rest])
        others = [j for j in range(3) if j != i]
        assert torch.equal(out[others], clean[others])
        c.v[page, row] = keep
