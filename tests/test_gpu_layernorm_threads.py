"""LayerNorm over rows called from several host threads with different widths: the bits of a call do not depend
on what other threads call, nor on the calls before it."""
import threading

import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("widths", [(8, 32), (72, 200), (40, 256, 129), (300, 500)])
@pytest.mark.parametrize("rows", [900, 9000])
def test_widths_of_one_kernel_from_several_threads(rows, widths):
    gen = torch.Generator(device="cuda").manual_seed(rows)

    class Call:
        def __init__(self, n):
            self.n, self.stream = n, torch.cuda.Stream()
            self.x, self.dy = (torch.randn(rows, n, generator=gen, device="cuda") for _ in range(2))
            self.size = B.layernorm_rows_bwd_scratch_bytes(rows, n)
            self.scratch = torch.empty(self.size, dtype=torch.uint8, device="cuda")

        def run(self, stream):
            n = self.n
            y, dx, mean, rstd, dg, db = self.out = [torch.empty_like(self.x), torch.empty_like(self.x)] + [
                torch.empty(m, device="cuda") for m in (rows, rows, n, n)]
            stream.wait_stream(torch.cuda.current_stream())
            B.layernorm_rows(self.x, None, None, y, mean, rstd, rows, n, n, n, B.F32, B.F32, stream=stream)
            B.layernorm_rows_bwd(self.dy, self.x, None, mean, rstd, dx, dg, db, rows, n, n, n, n, B.F32, B.F32, self.scratch,
                                 self.size, stream)
            stream.synchronize()
            return self.out

    calls = [Call(n) for n in widths]
    want = [[t.clone() for t in c.run(torch.cuda.current_stream())] for c in calls]
    wrong = []

    def work(i):
        for _ in range(50):
            if not all(torch.equal(a, b) for a, b in zip(calls[i].run(calls[i].stream), want[i])):
                wrong.append(widths[i])
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
