"""Waits that run out while copies and products are in flight: whichever role gives up first, a kernel waits for
what it has asked for before it ends, so the next call finds shared and tensor memory to itself."""
import subprocess
import sys
import time

import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_rows,heads", [(300, 2), (700, 40)])
def test_a_limit_far_too_short(q_rows, heads, dim):
    gen = torch.Generator(device="cuda").manual_seed(dim)
    make = lambda rows: torch.randn(2, rows, heads, dim, generator=gen, device="cuda").bfloat16()
    q, do, k, v = make(q_rows), make(q_rows), make(1500), make(1500)
    shape = B.XattnShape.of(q, k, v, q)
    nf, nb = B.xattn_fwd_scratch_bytes(shape), B.xattn_bwd_scratch_bytes(shape)
    scratch = torch.zeros(max(nf, nb, 16), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream()

    def step():
        o, dq, dk, dv = (torch.zeros_like(t) for t in (q, q, k, v))
        lse = torch.zeros(2, heads, q_rows, device="cuda")
        B.xattn_fwd(shape, q, k, v, None, o, lse, scratch, nf, stream)
        B.xattn_bwd(shape, q, k, v, None, o, lse, do, dq, dk, dv, scratch, nb, stream)
        return o, lse, dq, dk, dv
    want = step()
    assert B.device_status(stream)[0] == B.OK
    codes = []
    begin = time.perf_counter()
    try:
        B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 1)
        for _ in range(20):
            step()
            codes.append(B.device_status(stream)[0])
    finally:
        B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 0)
    took = time.perf_counter() - begin
    assert set(codes) <= {B.OK, B.ERR_DEVICE_TIMEOUT}
    print("gave up in", codes.count(B.ERR_DEVICE_TIMEOUT), "of", len(codes), "took", took)
    # (what is in flight lands in microseconds: a closing wait for what was never asked for would take two seconds)
    assert took < 2
    got = step()
    assert B.device_status(stream)[0] == B.OK
    assert all(torch.equal(a, b) for a, b in zip(want, got))


STATUS = r"""
import torch
from paper_2506_09092_b200 import binding as B
stream = torch.cuda.current_stream()
a, c = torch.ones(128, 128, device="cuda").bfloat16(), torch.empty(128, 128, device="cuda")
assert B.device_status(stream) == (B.OK, 0)                     # nothing has run
B.gemm_bf16(a, a, c, 128, 128, 128, 128, 128, 128, B.F32, stream)
assert B.device_status(stream) == (B.OK, 0) and bool((c == 128).all())
q = torch.randn(1, 40, 2, 64, device="cuda").bfloat16()
o, lse, dq = torch.empty_like(q), torch.empty(1, 2, 40, device="cuda"), torch.empty_like(q)
shape = B.XattnShape.of(q, q, q, o)
n = B.xattn_bwd_scratch_bytes(shape)
scratch = torch.empty(n, dtype=torch.uint8, device="cuda")
B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 1_000_000)
B.debug_set(B.DEBUG_SKIP_NEXT_XATTN_LOADS, 1)
B.xattn_fwd(shape, q, q, q, None, o, lse, None, 0, stream)
assert B.device_status(stream)[0] == B.ERR_DEVICE_TIMEOUT       # the first attention call gave up
assert B.device_status(stream) == (B.OK, 0)                     # reported once
B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 0)
B.xattn_fwd(shape, q, q, q, None, o, lse, None, 0, stream)
B.xattn_bwd(shape, q, q, q, None, o, lse, o, dq, None, None, scratch, n, stream)
assert B.device_status(stream) == (B.OK, 0) and bool(o.isfinite().all())
print("reported once")
"""


def test_status_before_and_after_the_first_attention_call():
    run = subprocess.run([sys.executable, "-c", STATUS], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "reported once" in run.stdout, run.stderr[-2000:]
