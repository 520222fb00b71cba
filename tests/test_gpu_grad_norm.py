"""The norm of a list of gradients and clipping, against 64 bits.

Tolerances: squares are rounded to 2^-24 of themselves and added eight at a time in fp32, so a
group's sum is off by at most 8 * 2^-24 and the norm, its root, by half of that, plus one
rounding: 5 * 2^-24.  A scaled gradient carries the coefficient's error (the norm's, a sum, a
quotient and the product: below 10 * 2^-24) and one rounding to its type."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def make(sizes, seed=0, scale=0.01, lead=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, (n, t) in enumerate(sizes):
        buf = torch.randn(n + lead, generator=g, device="cuda")
        out.append(((buf * scale * (1 + i % 5)).to(t))[lead:])
    return out


def scratch_for(table):
    n = B.grad_norm_scratch_bytes(table)
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n


def norm64(tensors):
    return float(torch.stack([(t.double() ** 2).sum() for t in tensors]).sum().sqrt()) if tensors else 0.0


def run_norm(tensors):
    table = B.tensor_table(tensors)
    scratch, n = scratch_for(table)
    norm = torch.full((1,), -1.0, device="cuda")
    B.grad_norm(table, norm, scratch, n, torch.cuda.current_stream())
    return float(norm)


F, H, BF = torch.float32, torch.float16, torch.bfloat16
LISTS = {
    "one": [(1, F)],
    "odd": [(1, BF), (2, H), (3, F), (7, BF), (9, H), (17, F), (2047, BF), (2049, H), (16385, F)],
    "empty among": [(0, F), (5, BF), (0, H), (100, F), (0, BF)],
    "large": [(5_000_011, BF), (3_000_001, F), (12345, H)],
    "64": [(100 + i, (F, BF, H)[i % 3]) for i in range(64)],
    "65": [(100 + i, (F, BF, H)[i % 3]) for i in range(65)],
    "many": [(1 + i % 300, (F, BF, H)[i % 3]) for i in range(2500)],
}


@pytest.mark.parametrize("name", list(LISTS))
@pytest.mark.parametrize("lead", [0, 1])
def test_norm_and_clip(name, lead):
    grads = make(LISTS[name], lead=lead)
    ref = norm64(grads)
    assert abs(run_norm(grads) - ref) <= 5 * U * ref
    for limit in (0.5 * ref, 2.0 * ref, 0.0):
        want = min(1.0, limit / (ref + 1e-6))
        outs = [torch.full_like(g, 7.0) for g in grads]
        inplace = [g.clone() for g in grads]
        results = []
        for tensors, dst in ((grads, outs), (inplace, None)):
            table = B.tensor_table(tensors, dst)
            scratch, n = scratch_for(table)
            norm = torch.full((1,), -1.0, device="cuda")
            B.grad_clip_norm(table, limit, 1e-6, norm, scratch, n, torch.cuda.current_stream())
            assert abs(float(norm) - ref) <= 5 * U * ref
            results.append(dst if dst is not None else tensors)
        split = [g.clone() for g in grads]                  # the two calls one after the other
        table = B.tensor_table(split)
        scratch, n = scratch_for(table)
        norm = torch.empty(1, device="cuda")
        B.grad_norm(table, norm, scratch, n, torch.cuda.current_stream())
        B.grad_clip(table, norm, limit, 1e-6, torch.cuda.current_stream())
        results.append(split)
        for g, a, b, c in zip(grads, *results):
            assert torch.equal(a, b) and torch.equal(a, c)
            if want == 1.0:
                assert torch.equal(a, g)
            exact = g.double() * want
            tol = exact.abs() * (torch.finfo(g.dtype).eps / 2 * (1 + 1e-3) + 10 * U) + (2.0 ** -25 if g.dtype == H else 1e-38)
            assert bool(((a.double() - exact).abs() <= tol).all())


def test_no_gradients():
    assert run_norm([]) == 0.0
    assert run_norm(make([(0, F), (0, BF)])) == 0.0
    table = B.tensor_table([])
    scratch, n = scratch_for(table)
    norm = torch.full((1,), 4.0, device="cuda")
    B.grad_clip_norm(table, 1.0, 1e-6, norm, scratch, n, torch.cuda.current_stream())
    assert float(norm) == 0.0


@pytest.mark.parametrize("scale", [1e-30, 1e-25, 1e-10, 1e10, 1e18, 3e30])
def test_norm_of_gradients_far_from_one(scale):
    g = make([(10001, F), (333, BF)], scale=scale)
    ref = norm64(g)
    assert abs(run_norm(g) - ref) <= 5 * U * ref
    mixed = g + make([(4097, F)], seed=5, scale=1e-5)       # and beside ordinary ones
    ref = norm64(mixed)
    assert abs(run_norm(mixed) - ref) <= 5 * U * ref


def test_zeros_and_non_finite_values():
    z = torch.zeros(50000, device="cuda", dtype=BF)
    assert run_norm([z]) == 0.0
    for bad, want in ((float("inf"), "inf"), (float("-inf"), "inf"), (float("nan"), "nan")):
        g = make([(5000, BF), (301, F)])
        g[1][300] = bad
        table = B.tensor_table(g)
        scratch, n = scratch_for(table)
        norm = torch.empty(1, device="cuda")
        B.grad_clip_norm(table, 1.0, 1e-6, norm, scratch, n, torch.cuda.current_stream())
        if want == "inf":
            assert float(norm) == float("inf")
            assert bool((g[0] == 0).all()) and bool((g[1][:300] == 0).all()) and bool(g[1][300].isnan())
        else:
            assert bool(norm.isnan().all())
            assert bool(g[0].isnan().all()) and bool(g[1].isnan().all())


def test_neighbours_are_untouched():
    buf = torch.full((64 + 1000 + 64,), 2.0, device="cuda", dtype=BF)
    for lead in range(8):
        part = buf[64 + lead:64 + lead + 901]
        part.copy_(torch.randn(901, device="cuda").to(BF))
        keep = part.clone()
        table = B.tensor_table([part])
        scratch, n = scratch_for(table)
        norm = torch.empty(1, device="cuda")
        B.grad_clip_norm(table, 1e-3, 0.0, norm, scratch, n, torch.cuda.current_stream())
        assert not torch.equal(part, keep)
        assert bool((buf[:64 + lead] == 2).all()) and bool((buf[64 + lead + 901:] == 2).all())
        buf.fill_(2.0)


def test_overlapping_outputs_are_refused():
    t = torch.zeros(100, device="cuda")
    u = torch.zeros(100, device="cuda")
    for tensors, outs in (([t, t], None), ([t, t[50:]], None), ([t[:50], t[40:]], None), ([t, u], [u, t]),
                          ([t[:50], t[50:]], [t[50:], u[:50]])):
        with pytest.raises(ValueError):
            B.tensor_table(tensors, outs)
    B.tensor_table([t[:50], t[50:]])
    B.tensor_table([t, t], [u, torch.zeros(100, device="cuda")])       # read twice, written apart
    with pytest.raises(ValueError):
        B.tensor_table([t.reshape(10, 10).t()])
    with pytest.raises(TypeError):
        B.tensor_table([t.double()])


def test_graph_replay_and_two_streams():
    grads = make([(70001, BF), (333, F), (4096, H)])
    ref = norm64(grads)
    outs = [torch.empty_like(g) for g in grads]
    table = B.tensor_table(grads, outs)
    norm = torch.empty(1, device="cuda")
    scratch, n = scratch_for(table)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.grad_clip_norm(table, 0.5, 1e-6, norm, scratch, n, torch.cuda.current_stream())
    side = torch.cuda.Stream()
    outs2 = [torch.empty_like(g) for g in grads]
    table2 = B.tensor_table(grads, outs2)
    norm2 = torch.empty(1, device="cuda")
    scratch2, _ = scratch_for(table2)
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        B.grad_clip_norm(table2, 0.5, 1e-6, norm2, scratch2, n, side)
    torch.cuda.synchronize()
    assert abs(float(norm) - ref) <= 5 * U * ref and float(norm) == float(norm2)
    assert all(torch.equal(a, b) for a, b in zip(outs, outs2))
    for g in grads:                       # new gradients in the same place: the replay sees them
        g.mul_(2)
    graph.replay()
    assert abs(float(norm) - norm64(grads)) <= 5 * U * norm64(grads)


def test_table_keeps_its_order_on_many_launches():
    """More tensors than one launch's list holds, the last one far larger than the rest."""
    grads = make([(3, F)] * 1500 + [(1_000_001, BF)])
    ref = norm64(grads)
    assert abs(run_norm(grads) - ref) <= 5 * U * ref
