"""Waits that run out while copies and products are in flight: whichever role gives up first, a kernel waits for
what it has asked for before it ends, so the next call finds shared and tensor memory to itself."""
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
