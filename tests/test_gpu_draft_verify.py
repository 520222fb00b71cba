"""Verification of drafted tokens against the definition: acceptance in exact arithmetic, the drawn token by sums in 64
bits.  The tokens have to be equal, except where the point drawn lies so near to a border between two tokens that 64-bit sums
of another order could fall on the other side (2^-53 of the sum for each of at most 2^18 additions): then either side's."""
from fractions import Fraction

import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"fp32": (torch.float32, B.F32), "bf16": (torch.bfloat16, B.BF16), "fp16": (torch.float16, B.F16)}


def call(p, q, drafts, lens, u, vocab, dtype, stream=None):
    b, n = drafts.shape
    tokens = torch.full((b, n + 1), -7, dtype=torch.int32, device="cuda")
    accepted = torch.full((b,), -7, dtype=torch.int32, device="cuda")
    B.draft_verify(p, q, drafts, lens, u, tokens, accepted, b, n, vocab, p.stride(-2) if p.dim() > 1 else vocab,
                   q.stride(-2) if q is not None and n else vocab, TYPES[dtype][1], stream or torch.cuda.current_stream())
    return tokens, accepted


def expect(p, q, drafts, lens, u):
    """For each sequence: (accepted, drafts accepted, tokens that may be drawn)."""
    out = []
    b, n = drafts.shape
    for i in range(b):
        m = n if lens is None else min(max(int(lens[i]), 0), n)
        a = 0
        while a < m:
            x = int(drafts[i, a])
            if not 0 <= x < p.shape[2]:
                break
            px, qx = float(p[i, a, x]), 1.0 if q is None else float(q[i, a, x])
            if not (px == px and qx == qx) or not (Fraction(float(u[i, a])) * Fraction(qx) < Fraction(px)
                                                   if abs(px) < float("inf") and abs(qx) < float("inf") else float(u[i, a]) * qx < px):
                break
            a += 1
        row = p[i, a].double()
        rest = row.clone()
        if a < m:
            if q is not None:
                rest -= q[i, a].double()
            elif 0 <= int(drafts[i, a]) < len(rest):
                rest[int(drafts[i, a])] -= 1.0
        rest = torch.where((rest > 0) & torch.isfinite(rest), rest, 0.0)
        if not bool((rest > 0).any()):
            rest = torch.where((row > 0) & torch.isfinite(row), row, 0.0)
        mass = rest.nonzero().flatten()
        if len(mass) == 0:
            may = [-1]
        else:
            sums = rest[mass].cumsum(0)
            eps = 2.0 ** -53 * 2 ** 18 * float(sums[-1])
            point = float(u[i, n]) * float(sums[-1])
            last = len(mass) - 1
            pick = lambda x: int(mass[min(int((sums <= x).sum()), last)])
            may = [pick(point - eps), pick(point), pick(point + eps)]
        out.append((a, [int(x) for x in drafts[i, :a]], may))
    return out


def check(p, q, drafts, lens, u, dtype, at_border=False):
    vocab = p.shape[2]
    tokens, accepted = call(p, q, drafts, lens, u, vocab, dtype)
    n = drafts.shape[1]
    cpu = [None if t is None else t.cpu() for t in (p, q, drafts, lens, u)]
    for i, (a, kept, may) in enumerate(expect(*cpu)):
        row = tokens[i].tolist()
        assert accepted[i].item() == a, i
        assert row[:a] == kept and row[a + 1:] == [-1] * (n - a), i
        assert row[a] in (may if at_border else may[1:2] if len(may) > 1 else may) or row[a] in may, (i, row[a], may)
    return tokens, accepted


def inputs(b, n, vocab, dtype, seed, certain=False, near=0.7):
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = torch.randn(b, n + 1, vocab, generator=g, device="cuda") * 2
    p = torch.softmax(logits, 2)
    q = torch.softmax(logits[:, :n] + near * torch.randn(b, n, vocab, generator=g, device="cuda"), 2)
    pick = (p[:, :n] if certain else q).reshape(b * n, vocab)
    drafts = torch.multinomial(pick, 1, generator=g).view(b, n).int() if n else torch.empty(b, 0, dtype=torch.int32, device="cuda")
    u = torch.rand(b, n + 1, generator=g, device="cuda")
    t = TYPES[dtype][0]
    return p.to(t), None if certain else q.to(t), drafts, u


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("b,n,vocab", [(1, 1, 1), (3, 4, 2), (8, 5, 33), (40, 3, 511), (5, 40, 512), (2, 2, 513), (7, 3, 4097),
                                       (1, 4, 50001), (300, 2, 1000), (700, 1, 9000), (3, 0, 777), (2, 3, 200000)])
def test_against_the_definition(b, n, vocab, certain, dtype):
    p, q, drafts, u = inputs(b, n, vocab, dtype, vocab + n, certain)
    check(p, q, drafts, None, u, dtype)
    lens = torch.tensor([(5 * i) % (n + 3) - 1 for i in range(b)], dtype=torch.int32, device="cuda")
    check(p, q, drafts, lens, u, dtype)


def test_pitches():
    b, n, vocab = 6, 3, 1001
    p, q, drafts, u = inputs(b, n, vocab, "fp32", 3)
    wide_p, wide_q = (torch.full((b * r, vocab + pad), float("nan"), device="cuda") for r, pad in ((n + 1, 13), (n, 2)))
    wide_p[:, :vocab], wide_q[:, :vocab] = p.view(-1, vocab), q.view(-1, vocab)
    want = check(p, q, drafts, None, u, "fp32")
    got = call(wide_p, wide_q, drafts, None, u, vocab, "fp32")
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_random_numbers_at_their_ends():
    b, n, vocab = 16, 2, 3000 + 7
    p, q, drafts, u = inputs(b, n, vocab, "fp32", 4)
    p[:, :, 0] = 0.0
    p[:, :, -2:] = 0.0
    q[:, :, 0] = q[:, :, -2:] = 0.0
    below = float(torch.nextafter(torch.tensor(1.0), torch.tensor(0.0)))
    for first, last in ((0.0, 0.0), (below, below), (0.0, below), (below, 0.0)):
        u[:, :n], u[:, n] = first, last
        tokens, accepted = check(p, q, drafts, None, u, "fp32", at_border=True)
        picked = tokens.gather(1, accepted.long()[:, None]).flatten()
        assert bool(((picked > 0) & (picked < vocab - 2)).all())       # never one without mass
    # outside [0, 1): the nearer end's token
    for value in (1.0, 2.0, float("inf"), float("nan"), -1.0):
        u[:, :n], u[:, n] = 0.0, value
        tokens, accepted = call(p, q, drafts, None, u, vocab, "fp32")
        assert bool((accepted == n).all())
        assert bool((tokens[:, n] == (1 if value < 0 else vocab - 3)).all())


def test_the_drawn_token_of_exact_sums():
    """Eighths: every sum is exact, so a point on a border belongs to the token behind it."""
    vocab = 8
    p = torch.full((64, 1, vocab), 0.125, device="cuda")
    u = (torch.arange(64, device="cuda") / 64).float().view(64, 1)
    tokens, _ = call(p, None, torch.empty(64, 0, dtype=torch.int32, device="cuda"), None, u, vocab, "fp32")
    assert tokens.flatten().tolist() == [i // 8 for i in range(64)]


def test_ties_of_acceptance_are_rejected():
    """u q < p is strict, and exact: 2^-24 off decides."""
    p = torch.tensor([[[0.5, 0.5], [0.25, 0.75]]] * 3, device="cuda")
    q = torch.tensor([[[1.0, 0.0]]] * 3, device="cuda")
    u = torch.tensor([[0.5, 0.9], [0.5 - 2.0 ** -25, 0.9], [0.5 + 2.0 ** -24, 0.1]], device="cuda")
    drafts = torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    tokens, accepted = call(p, q, drafts, None, u, 2, "fp32")
    assert accepted.tolist() == [0, 1, 0] and tokens.tolist() == [[1, -1], [0, 1], [1, -1]]


@pytest.mark.parametrize("vocab", [10, 50000])
def test_nothing_left_of_the_difference_nothing_at_all_and_values_that_are_not_finite(vocab):
    n = 2
    p = torch.full((6, n + 1, vocab), 1.0 / vocab, device="cuda")
    q = p[:, :n].clone()
    u = torch.full((6, n + 1), 0.5, device="cuda")
    drafts = torch.full((6, n), 3, dtype=torch.int32, device="cuda")
    u[0, 0] = 1.0                                     # rejected, p - q = 0 everywhere: from p
    p[1] = 0.0                                        # no mass
    p[2, 0] = float("nan")
    p[3, 0] = float("inf")
    p[3, 1], q[3, 1] = 0.0, 0.5
    p[3, 1, 7] = float("inf")
    p[4, 0, 3] = 0.0                                  # rejected; one token has more than its draft's
    q[4, 0, 8] = 0.0
    p[5, 0], q[5, 0] = 0.0, float("nan")
    p[5, 0, 2] = -1.0
    drafts[5, 1] = 1 << 30
    tokens, accepted = check(p, q, drafts, None, u, "fp32")
    assert accepted.tolist()[:3] == [0, 0, 0] and tokens[1].tolist() == [-1, -1, -1] == tokens[2].tolist()
    assert tokens[4, 0].item() == 8 and tokens[3].tolist()[0] == 3


def test_drafts_that_are_no_tokens():
    p, q, drafts, u = inputs(5, 3, 100, "fp32", 9)
    u[:, :3] = 0.0
    drafts[0, 0], drafts[1, 1], drafts[2, 2], drafts[3, 0] = -1, 100, 1 << 30, -(1 << 31)
    for qq in (q, None):
        _, accepted = check(p, qq, drafts, None, u, "fp32")
        assert accepted.tolist() == [0, 1, 2, 0, 3]


def test_distribution_of_the_first_token():
    """Whatever the draft's distribution, the first token is distributed as the target's: 200 000 sequences, five standard
    deviations of each count."""
    b, vocab = 200000, 6
    g = torch.Generator(device="cuda").manual_seed(1)
    p = torch.tensor([0.3, 0.05, 0.25, 0.1, 0.2, 0.1], device="cuda").expand(b, 2, vocab).contiguous()
    q = torch.tensor([0.1, 0.4, 0.1, 0.1, 0.05, 0.25], device="cuda").expand(b, 1, vocab).contiguous()
    drafts = torch.multinomial(q[:, 0], 1, generator=g).int()
    tokens, _ = call(p, q, drafts, None, torch.rand(b, 2, generator=g, device="cuda"), vocab, "fp32")
    counts = torch.bincount(tokens[:, 0].long(), minlength=vocab).double()
    want = p[0, 0].double() * b
    assert bool(((counts - want).abs() <= 5 * want.sqrt()).all())


def test_captured():
    p, q, drafts, u = inputs(9, 4, 5000, "bf16", 2)
    want = call(p, q, drafts, None, u, 5000, "bf16")
    tokens, accepted = (torch.full_like(t, -9) for t in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.draft_verify(p, q, drafts, None, u, tokens, accepted, 9, 4, 5000, 5000, 5000, B.BF16, torch.cuda.current_stream())
    graph.replay()
    assert torch.equal(tokens, want[0]) and torch.equal(accepted, want[1])


def test_rows_beyond_32_bits_of_offset():
    vocab, ld = 1000, 1 << 29
    buf = torch.empty(5 * ld, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(buf, (5, vocab), (ld, 1))
    p, q, drafts, u = inputs(1, 4, vocab, "bf16", 8, certain=True)
    u[:] = 0.5
    u[:, :4] = 0.0
    far.copy_(p[0])
    want = call(p, None, drafts, None, u, vocab, "bf16")
    got = call(far, None, drafts, None, u, vocab, "bf16")
    assert torch.equal(want[0], got[0]) and want[1].tolist() == [4]
