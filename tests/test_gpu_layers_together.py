"""The layer operators as a program uses them: a block that attends to an encoder's states, trained
for one step (normalise, project, attend, project, all gradients, clip) with the library's own
products in between, and the same block answering with single tokens.

The step's results are compared with 64-bit automatic differentiation of the same block.  Along the
longest path (gamma's gradient: input, normalised input, Q, K, P, O, its gradient, dS, dQ, the
projection's gradient) ten tensors are rounded to bf16; a rounding is at most 2^-8 of each value, so of
the tensor's 2-norm, and the scores (at most about 1.5 in size here) pass theirs on to the
probabilities at most 1.5 times as large: 15 * 2^-8 = 6 % of the norm if all pointed one way."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
BATCH, QL, KL, DIM, HEADS, KV_HEADS, HEAD = 3, 70, 150, 256, 4, 2, 64
LENS = [150, 37, 129]


def product(a, b, out_f32=False):
    """a b for bf16 matrices through the library."""
    (m, k), n = a.shape, b.shape[1]
    c = torch.empty(m, n, dtype=torch.float32 if out_f32 else BF, device="cuda")
    a, b = a.contiguous(), b.contiguous()
    B.gemm_bf16(a, b, c, m, n, k, k, n, n, B.F32 if out_f32 else B.BF16, torch.cuda.current_stream())
    return c


class Block:
    """Weights, and the buffers and plans that a program sets up once."""

    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.x, self.enc = rnd(BATCH * QL, DIM).to(BF), rnd(BATCH * KL, DIM).to(BF)
        self.gamma, self.beta = 1 + 0.1 * rnd(DIM), 0.1 * rnd(DIM)
        self.wq = (rnd(DIM, HEADS * HEAD) * DIM ** -0.5 * 0.3).to(BF)
        self.wkv = (rnd(DIM, 2 * KV_HEADS * HEAD) * DIM ** -0.5).to(BF)
        self.wo = (rnd(HEADS * HEAD, DIM) * DIM ** -0.5).to(BF)
        self.dout = rnd(BATCH * QL, DIM).to(BF)                  # the loss is sum(out * dout)
        self.lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
        rows = BATCH * QL
        self.xn, self.mean, self.rstd = torch.empty_like(self.x), *torch.empty(2, rows, device="cuda")
        self.o = torch.empty(BATCH, QL, HEADS, HEAD, dtype=BF, device="cuda")
        self.lse = torch.empty(BATCH, HEADS, QL, device="cuda")
        self.dq = torch.empty_like(self.o)
        self.dkv = torch.empty(BATCH, KL, 2, KV_HEADS, HEAD, dtype=BF, device="cuda")
        self.dx, self.dgamma, self.dbeta = torch.empty_like(self.x), torch.empty(DIM, device="cuda"), torch.empty(DIM, device="cuda")
        self.norm = torch.empty(1, device="cuda")
        self.ln_bytes = B.layernorm_rows_bwd_scratch_bytes(rows, DIM)
        self.ln_scratch = torch.empty(self.ln_bytes, dtype=torch.uint8, device="cuda")
        self.att_scratch = None

    def forward(self, stream):
        rows = BATCH * QL
        B.layernorm_rows(self.x, self.gamma, self.beta, self.xn, self.mean, self.rstd, rows, DIM, DIM, DIM, B.BF16, B.F32,
                         1e-5, stream)
        self.q = product(self.xn, self.wq).view(BATCH, QL, HEADS, HEAD)
        self.kv = product(self.enc, self.wkv).view(BATCH, KL, 2, KV_HEADS, HEAD)
        k, v = self.kv[:, :, 0], self.kv[:, :, 1]
        self.shape = B.XattnShape.of(self.q, k, v, self.o)
        if self.att_scratch is None:
            self.fwd_bytes, self.bwd_bytes = B.xattn_fwd_scratch_bytes(self.shape), B.xattn_bwd_scratch_bytes(self.shape)
            self.att_scratch = torch.empty(max(self.fwd_bytes, self.bwd_bytes), dtype=torch.uint8, device="cuda")
        B.xattn_fwd(self.shape, self.q, k, v, self.lens, self.o, self.lse, self.att_scratch, self.fwd_bytes, stream)
        self.out = product(self.o.view(rows, -1), self.wo)

    def backward(self, stream, limit):
        rows = BATCH * QL
        self.dwo = product(self.o.view(rows, -1).t(), self.dout)
        do = product(self.dout, self.wo.t()).view(BATCH, QL, HEADS, HEAD)
        k, v = self.kv[:, :, 0], self.kv[:, :, 1]
        B.xattn_bwd(self.shape, self.q, k, v, self.lens, self.o, self.lse, do, self.dq, self.dkv[:, :, 0], self.dkv[:, :, 1],
                    self.att_scratch, self.bwd_bytes, stream)
        dq, dkv = self.dq.view(rows, -1), self.dkv.view(BATCH * KL, -1)
        self.dwq, self.dwkv = product(self.xn.t(), dq), product(self.enc.t(), dkv)
        dxn = product(dq, self.wq.t())
        B.layernorm_rows_bwd(dxn, self.x, self.gamma, self.mean, self.rstd, self.dx, self.dgamma, self.dbeta, rows, DIM, DIM, DIM,
                             DIM, B.BF16, B.F32, self.ln_scratch, self.ln_bytes, stream)
        self.table = B.tensor_table([self.dwq, self.dwkv, self.dwo, self.dgamma, self.dbeta])
        n = B.grad_norm_scratch_bytes(self.table)
        self.clip_scratch = torch.empty(n, dtype=torch.uint8, device="cuda")
        B.grad_clip_norm(self.table, limit, 1e-6, self.norm, self.clip_scratch, n, stream)

    def results(self):
        return dict(out=self.out, dx=self.dx, dwq=self.dwq, dwkv=self.dwkv, dwo=self.dwo, dgamma=self.dgamma, dbeta=self.dbeta,
                    norm=self.norm)


def reference(b):
    """The same block and its gradients by 64-bit automatic differentiation."""
    leaf = lambda t: t.double().requires_grad_()
    x, gamma, beta, wq, wkv, wo = (leaf(t) for t in (b.x, b.gamma, b.beta, b.wq, b.wkv, b.wo))
    xc = x - x.mean(1, keepdim=True)
    xn = xc / torch.sqrt((xc * xc).mean(1, keepdim=True) + 1e-5) * gamma + beta
    q = (xn @ wq).view(BATCH, QL, HEADS, HEAD).transpose(1, 2)
    kv = (b.enc.double() @ wkv).view(BATCH, KL, 2, KV_HEADS, HEAD)
    k, v = (kv[:, :, i].transpose(1, 2).repeat_interleave(HEADS // KV_HEADS, 1) for i in (0, 1))
    pad = torch.arange(KL, device="cuda")[None, :] >= b.lens[:, None]
    s = (q @ k.transpose(2, 3) * HEAD ** -0.5).masked_fill(pad[:, None, None, :], float("-inf"))
    out = (torch.softmax(s, 3) @ v).transpose(1, 2).reshape(BATCH * QL, -1) @ wo
    (out * b.dout.double()).sum().backward()
    return out.detach(), dict(dx=x.grad, dwq=wq.grad, dwkv=wkv.grad, dwo=wo.grad, dgamma=gamma.grad, dbeta=beta.grad)


def off_by(got, want):
    return float((got.double() - want).norm() / want.norm())


def test_training_step():
    b = Block(1)
    out, grads = reference(b)
    norm = float(torch.stack([grads[k].square().sum() for k in ("dwq", "dwkv", "dwo", "dgamma", "dbeta")]).sum().sqrt())
    limit = 0.25 * norm
    b.forward(torch.cuda.current_stream())
    b.backward(torch.cuda.current_stream(), limit)
    assert B.device_status(torch.cuda.current_stream())[0] == B.OK
    bound = 15 * 2.0 ** -8
    assert off_by(b.out, out) < bound
    assert abs(float(b.norm) / norm - 1) < bound
    for name, want in grads.items():
        scale = 1.0 if name == "dx" else limit / norm                # the weights' gradients were clipped
        assert off_by(b.results()[name], want * scale) < 2 * bound, name


def test_training_step_as_a_graph_beside_an_eager_one():
    """The captured step replayed while the same step of other weights runs on another stream (which has a
    workspace of its own for the products)."""
    first, second = Block(1), Block(2)
    stream = torch.cuda.current_stream()
    eager = []
    for b in (first, second):
        b.forward(stream)
        b.backward(stream, 1.0)
        eager.append({k: v.clone() for k, v in b.results().items()})
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        first.forward(torch.cuda.current_stream())
        first.backward(torch.cuda.current_stream(), 1.0)
    workspace = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    B.set_workspace_for_stream(side, workspace, workspace.numel())
    try:
        side.wait_stream(stream)
        for _ in range(3):
            graph.replay()
            with torch.cuda.stream(side):
                second.forward(side)
                second.backward(side, 1.0)
        torch.cuda.synchronize()
    finally:
        B.set_workspace_for_stream(side, None, 0)
    for b, want in zip((first, second), eager):
        for k, v in b.results().items():
            tol = 0.0 if b is first else 2.0 ** -7                   # (the side stream's products may be split otherwise)
            assert off_by(v, want[k].double()) <= tol, k


def test_single_tokens_answer_like_the_whole_sequence():
    b = Block(3)
    stream = torch.cuda.current_stream()
    b.forward(stream)
    k, v = b.kv[:, :, 0], b.kv[:, :, 1]
    for pos in (0, 33, QL - 1):
        x = b.x.view(BATCH, QL, DIM)[:, pos].contiguous()
        xn, o = torch.empty_like(x), torch.empty(BATCH, 1, HEADS, HEAD, dtype=BF, device="cuda")
        B.layernorm_rows(x, b.gamma, b.beta, xn, None, None, BATCH, DIM, DIM, DIM, B.BF16, B.F32, 1e-5, stream)
        # at most two fp32 sums in another order before the rounding: one step of bf16
        assert bool(((xn.float() - b.xn.view(BATCH, QL, DIM)[:, pos].float()).abs() <= 2.0 ** -7 * xn.float().abs() + 1e-6).all())
        q = b.q[:, pos:pos + 1].contiguous()
        shape = B.XattnShape.of(q, k, v, o)
        n = B.xattn_fwd_scratch_bytes(shape)
        scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        B.xattn_fwd(shape, q, k, v, b.lens, o, None, scratch, n, stream)
        whole = b.o[:, pos:pos + 1].float()
        # each of the two within 2^-8 (|O| + sum p |v|) of the exact value, sum p |v| <= max |v| of the item
        top = v.float().abs().amax((1, 3)).repeat_interleave(HEADS // KV_HEADS, 1)[:, None, :, None]
        assert bool(((o.float() - whole).abs() <= 2 * 2.0 ** -8 * (whole.abs() + top)).all())


@pytest.mark.parametrize("task,size", [("ln-rows", 50), ("ln-rows-bwd", 50), ("grad-clip", 10000), ("xattn", 64), ("xattn-token", 100),
                                       ("xattn-bwd", 64)])
def test_harness_layer_commands_run(task, size, capsys):
    import json
    from paper_2506_09092_b200 import harness as H
    H._main(["--task", task, "--size", str(size), "--iters", "2", "--warmup", "1"])
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["task"] == task and line["status"] == 0 and line["us_median"] > 0
