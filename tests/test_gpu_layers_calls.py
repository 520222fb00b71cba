"""Calls of the layer operators that other tests do not make: the very first call of a process inside
a stream capture, calls that overlap on two streams, operands without rows whose strides mean nothing."""
import ctypes
import subprocess
import sys

import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu

FIRST = r"""
import sys, torch
from paper_2506_09092_b200 import binding as B
what = sys.argv[1]
torch.manual_seed(0)
stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
if what in ("xattn", "token"):
    rows = 130 if what == "xattn" else 1
    q, do = (torch.randn(2, rows, 4, 64, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn(2, 300, 4, 64, device="cuda").bfloat16() for _ in range(2))
    o, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, v))
    lse = torch.empty(2, 4, rows, device="cuda")
    shape = B.XattnShape.of(q, k, v, o)
    nf, nb = B.xattn_fwd_scratch_bytes(shape), B.xattn_bwd_scratch_bytes(shape)
    sf, sb = (torch.empty(max(n, 16), dtype=torch.uint8, device="cuda") for n in (nf, nb))
    def call():
        B.xattn_fwd(shape, q, k, v, None, o, lse, sf, nf, torch.cuda.current_stream())
        B.xattn_bwd(shape, q, k, v, None, o, lse, do, dq, dk, dv, sb, nb, torch.cuda.current_stream())
    outs = (o, lse, dq, dk, dv)
elif what == "ln":
    x, dy = (torch.randn(700, 1000, device="cuda") for _ in range(2))
    y, dx, dg, db = torch.empty_like(x), torch.empty_like(x), torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
    mean, rstd = torch.empty(700, device="cuda"), torch.empty(700, device="cuda")
    n = B.layernorm_rows_bwd_scratch_bytes(700, 1000)
    scr = torch.empty(n, dtype=torch.uint8, device="cuda")
    def call():
        s = torch.cuda.current_stream()
        B.layernorm_rows(x, None, None, y, mean, rstd, 700, 1000, 1000, 1000, B.F32, B.F32, stream=s)
        B.layernorm_rows_bwd(dy, x, None, mean, rstd, dx, dg, db, 700, 1000, 1000, 1000, 1000, B.F32, B.F32, scr, n, stream=s)
    outs = (y, mean, rstd, dx, dg, db)
else:
    g = [torch.randn(5000, device="cuda").bfloat16(), torch.randn(77, device="cuda")]
    out = [torch.empty_like(t) for t in g]
    table, norm = B.tensor_table(g, out), torch.empty(1, device="cuda")
    n = B.grad_norm_scratch_bytes(table)
    scr = torch.empty(n, dtype=torch.uint8, device="cuda")
    def call():
        B.grad_clip_norm(table, 1.0, 1e-6, norm, scr, n, torch.cuda.current_stream())
    outs = (*out, norm)
torch.cuda.synchronize()
with torch.cuda.graph(graph, stream=stream):
    call()
for t in outs:
    t.fill_(7)
graph.replay()
torch.cuda.synchronize()
first = [t.clone() for t in outs]
assert all(bool(torch.isfinite(t).all()) for t in first)
for t in outs:
    t.fill_(9)
call()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(first, outs))
assert B.device_status(torch.cuda.current_stream())[0] == B.OK
print("captured first")
"""


@pytest.mark.parametrize("what", ["xattn", "token", "ln", "clip"])
def test_first_call_of_a_process_is_captured(what):
    run = subprocess.run([sys.executable, "-c", FIRST, what], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "captured first" in run.stdout, run.stderr[-2000:]


def test_attention_calls_overlap_on_two_streams():
    gen = torch.Generator(device="cuda").manual_seed(3)
    sides, sets = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for rows, states, heads, dim in ((700, 900, 6, 128), (3, 2100, 4, 64)):
        q, do = (torch.randn(2, rows, heads, dim, generator=gen, device="cuda").half() for _ in range(2))
        k, v = (torch.randn(2, states, heads // 2, dim, generator=gen, device="cuda").half() for _ in range(2))
        outs = [torch.empty_like(t) for t in (q, q, k, v)] + [torch.empty(2, heads, rows, device="cuda")]
        shape = B.XattnShape.of(q, k, v, outs[0])
        lens = torch.tensor([states, states // 3], dtype=torch.int32, device="cuda")
        nf, nb = B.xattn_fwd_scratch_bytes(shape), B.xattn_bwd_scratch_bytes(shape)
        scr = [torch.empty(max(n, 16), dtype=torch.uint8, device="cuda") for n in (nf, nb)]

        def call(stream, shape=shape, q=q, k=k, v=v, do=do, outs=outs, lens=lens, nf=nf, nb=nb, scr=scr):
            o, dq, dk, dv, lse = outs
            B.xattn_fwd(shape, q, k, v, lens, o, lse, scr[0], nf, stream)
            B.xattn_bwd(shape, q, k, v, lens, o, lse, do, dq, dk, dv, scr[1], nb, stream)
        sets.append((call, outs))
    want = []
    for call, outs in sets:
        call(torch.cuda.current_stream())
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
        for t in outs:
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(10):
        for (call, _o), side in zip(sets, sides):
            call(side)
    torch.cuda.synchronize()
    for (_c, outs), w in zip(sets, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, w))
    assert B.device_status(torch.cuda.current_stream())[0] == B.OK


@pytest.mark.parametrize("bad", [0, 3, -8])
@pytest.mark.parametrize("q_rows", [1, 100])
def test_strides_of_operands_without_rows_do_not_matter(q_rows, bad):
    q, do = (torch.randn(2, q_rows, 32, 64, device="cuda").bfloat16() for _ in range(2))
    o, dq = torch.full_like(q, 7), torch.full_like(q, 7)
    lse = torch.empty(2, 32, q_rows, device="cuda")
    st, none = (ctypes.c_int64 * 3)(*q.stride()[:3]), (ctypes.c_int64 * 3)(bad, bad, bad)
    shape = B.XattnShape(batch=2, q_rows=q_rows, kv_rows=0, q_heads=32, kv_heads=4, head_dim=64, dtype=B.BF16, scale=0.125,
                         q_stride=st, k_stride=none, v_stride=none, o_stride=st)
    n = B.xattn_bwd_scratch_bytes(shape)
    scr = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.xattn_fwd(shape, q, None, None, None, o, lse, None, 0, torch.cuda.current_stream())
    B.xattn_bwd(shape, q, None, None, None, o, lse, do, dq, None, None, scr, n, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert not o.any() and not dq.any() and bool((lse == float("-inf")).all())
    # and no queries: the states' gradients are zero whatever the queries' strides say
    dk, dv = (torch.full((2, 50, 4, 64), 7, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    kst = (ctypes.c_int64 * 3)(*dk.stride()[:3])
    shape = B.XattnShape(batch=2, q_rows=0, kv_rows=50, q_heads=32, kv_heads=4, head_dim=64, dtype=B.BF16, scale=0.125,
                         q_stride=none, k_stride=kst, v_stride=kst, o_stride=none)
    k, v = torch.randn_like(dk), torch.randn_like(dv)
    B.xattn_bwd(shape, None, k, v, None, None, None, None, None, dk, dv, None, 0, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert not dk.any() and not dv.any()


@pytest.mark.parametrize("max_norm,eps,value", [(0.0, 0.0, 0.0), (float("inf"), 1e-6, float("inf")),
                                                (0.0, 0.0, 2.0), (float("inf"), 0.0, float("nan"))])
def test_clip_limits_at_both_ends(max_norm, eps, value):
    """No limit leaves gradients alone whatever their norm, a limit of zero leaves zeros at zero."""
    g = torch.tensor([0.0, 1.0 if value else 0.0, value], device="cuda")
    out = torch.full_like(g, 7)
    table, norm = B.tensor_table([g], [out]), torch.empty(1, device="cuda")
    n = B.grad_norm_scratch_bytes(table)
    scr = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.grad_clip_norm(table, max_norm, eps, norm, scr, n, torch.cuda.current_stream())
    if value != value:
        assert bool(out.isnan().all())
    else:
        want = torch.zeros_like(g) if max_norm == 0 else g
        assert torch.equal(out, want)


STRIDE = 1 << 23            # 300 rows of it: the last lies 2.5e9 elements into its buffer


def far_rows(buf, rows, cols, at):
    return torch.as_strided(buf, (rows, cols), (STRIDE, 1), at)


def test_attention_gradients_with_more_than_32_bits_of_offset():
    rows, dim = 300, 64
    ops = torch.empty(rows * STRIDE, dtype=torch.bfloat16, device="cuda")
    res = torch.empty_like(ops)
    gen = torch.Generator(device="cuda").manual_seed(5)

    def far(buf, at):
        return far_rows(buf, rows, dim, at).view(1, rows, 1, dim)
    q, k, v, do, o = (far(ops, 4096 * i) for i in range(5))
    for t in (q, k, v, do):
        t.copy_(torch.randn(1, rows, 1, dim, generator=gen, device="cuda"))
    dq, dk, dv = (far(res, 4096 * i) for i in range(3))

    def run(q, k, v, do, o, dq, dk, dv):
        lse = torch.empty(1, 1, rows, device="cuda")
        shape = B.XattnShape.of(q, k, v, o)
        nf, nb = B.xattn_fwd_scratch_bytes(shape), B.xattn_bwd_scratch_bytes(shape)
        scr = torch.empty(max(nf, nb), dtype=torch.uint8, device="cuda")
        B.xattn_fwd(shape, q, k, v, None, o, lse, scr, nf, torch.cuda.current_stream())
        B.xattn_bwd(shape, q, k, v, None, o, lse, do, dq, dk, dv, scr, nb, torch.cuda.current_stream())
        return o, dq, dk, dv
    near = [t.contiguous() for t in (q, k, v, do)] + [torch.empty(1, rows, 1, dim, dtype=torch.bfloat16, device="cuda")
                                                       for _ in range(4)]
    for a, b in zip(run(q, k, v, do, o, dq, dk, dv), run(*near)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n", [200, 4096, 4097, 20000])
def test_layernorm_rows_with_more_than_32_bits_of_offset(n):
    rows = 300
    buf = torch.empty(rows * STRIDE, dtype=torch.float16, device="cuda")
    x, dy, y, dx = (far_rows(buf, rows, n, 65536 * i) for i in range(4))
    for t in (x, dy):
        t.copy_(torch.randn(rows, n, device="cuda"))

    def run(x, dy, y, dx):
        ld = x.stride(0)
        mean, rstd, dg, db = (torch.empty(m, device="cuda") for m in (rows, rows, n, n))
        size = B.layernorm_rows_bwd_scratch_bytes(rows, n)
        scr, s = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.cuda.current_stream()
        B.layernorm_rows(x, None, None, y, mean, rstd, rows, n, ld, ld, B.F16, B.F32, stream=s)
        B.layernorm_rows_bwd(dy, x, None, mean, rstd, dx, dg, db, rows, n, ld, ld, ld, B.F16, B.F32, scr, size, stream=s)
        return y, mean, rstd, dx, dg, db
    near = [x.contiguous(), dy.contiguous(), torch.empty(rows, n, dtype=torch.float16, device="cuda"),
            torch.empty(rows, n, dtype=torch.float16, device="cuda")]
    for a, b in zip(run(x, dy, y, dx), run(*near)):
        assert torch.equal(a, b)


def test_gradient_of_more_than_32_bits_of_elements():
    n = (1 << 32) + 77
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    table, norm = B.tensor_table([g]), torch.empty(1, device="cuda")
    size = B.grad_norm_scratch_bytes(table)
    scr = torch.empty(size, dtype=torch.uint8, device="cuda")
    want = 0.5 * n ** 0.5
    # the norm is exact but for its last rounding: every partial sum is a multiple of 1/4 below 2^53
    B.grad_clip_norm(table, want / 4, 0.0, norm, scr, size, torch.cuda.current_stream())
    assert abs(norm.item() - want) <= want * 2.0 ** -23
    # c is off from 1/4 by at most a few 2^-24, far below half a step of bf16
    lo, hi = torch.aminmax(g)
    assert lo.item() == hi.item() == 0.125


@pytest.mark.parametrize("count", [3, 70])
@pytest.mark.parametrize("lead", [0, 1])
def test_clip_of_many_elements_equals_the_formula(count, lead):
    """More than 17 million elements: the same fp32 quotient, product and rounding as elementwise code."""
    types = (torch.float32, torch.bfloat16, torch.float16)
    gen = torch.Generator(device="cuda").manual_seed(count)
    size = 24_000_000 // count
    bufs = [torch.randn(size + 13 * i + 8, generator=gen, device="cuda").to(types[i % 3]) for i in range(count)]
    grads = [b[lead:lead + size + 13 * i] for i, b in enumerate(bufs)]
    norm = torch.empty(1, device="cuda")
    for shift in (0, 1, None):                   # beside, off by one element, in place
        if shift is None:
            keep = [b.clone() for b in bufs]
            src = out = [b[lead:lead + g.numel()] for b, g in zip(keep, grads)]
        else:
            keep = [torch.full((b.numel() + 8,), 7.0, dtype=b.dtype, device="cuda") for b in bufs]
            src, out = grads, [b[lead + shift:lead + shift + g.numel()] for b, g in zip(keep, grads)]
        table = B.tensor_table(src, out)
        n = B.grad_norm_scratch_bytes(table)
        scr = torch.empty(n, dtype=torch.uint8, device="cuda")
        B.grad_clip_norm(table, 3.0, 1e-6, norm, scr, n, torch.cuda.current_stream())
        # (a number divided by a tensor is its reciprocal times the number: rounded twice)
        coef = torch.full_like(norm, 3.0) / (norm + 1e-6)
        for g, o, b in zip(grads, out, keep):
            assert torch.equal(o, (g.float() * coef).to(g.dtype))
            if shift is not None:
                first = lead + shift
                assert bool((b[:first] == 7).all()) and bool((b[first + g.numel():] == 7).all())
