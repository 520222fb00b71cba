"""The paged cache as an answering program uses it: prompts, then steps of drafted tokens that are verified and given back, through two
attention layers with the library's own products; sequences that fork, end and are compacted on the way.

Attention is compared with the dense formula in 64 bits on the same (rounded) queries, keys and values: each result is within
h (|O| + sum p |v|) + small terms of it, h half a step of bf16, so 2.1 h (|O| + max |v|) is a bound."""
import pytest
import torch

from page_book import Book
from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
LAYERS, DIM, HQ, HK, HEAD, ROWS, VOCAB, DRAFTS = 2, 256, 8, 2, 64, 8, 500, 3
H = 2.0 ** -8


def product(a, b, out_f32=False):
    (m, k), n = a.shape, b.shape[1]
    c = torch.empty(m, n, dtype=torch.float32 if out_f32 else BF, device="cuda")
    B.gemm_bf16(a.contiguous(), b.contiguous(), c, m, n, k, k, n, n, B.F32 if out_f32 else B.BF16, torch.cuda.current_stream())
    return c


class Server:
    """`slots` sequences, each layer's pools, and every token with its keys and values as they were written."""

    def __init__(self, slots, pages, cols, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.gen = g
        self.embed = rnd(VOCAB, DIM).to(BF)
        self.wqkv = [(rnd(DIM, (HQ + 2 * HK) * HEAD) * DIM ** -0.5).to(BF) for _ in range(LAYERS)]
        self.wo = [(rnd(HQ * HEAD, DIM) * (HQ * HEAD) ** -0.5).to(BF) for _ in range(LAYERS)]
        self.pools = [torch.full((pages, 2, ROWS, HK, HEAD), float("nan"), dtype=BF, device="cuda") for _ in range(LAYERS)]
        self.page_pools = B.page_pools(self.pools)
        self.book, self.want = B.PageBook(pages, ROWS, slots, cols), Book(pages, ROWS, slots, cols)
        self.result = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.need = max(B.pages_resize_scratch_bytes(self.book, slots), B.pages_fork_scratch_bytes(self.book, slots),
                        B.pages_compact_scratch_bytes(self.book))
        self.scratch = torch.empty(self.need, dtype=torch.uint8, device="cuda")
        self.keys = [[torch.empty(0, HK, HEAD, dtype=BF, device="cuda") for _ in range(LAYERS)] for _ in range(slots)]
        self.values = [list(k) for k in self.keys]
        self.tokens = [[] for _ in range(slots)]

    def ints(self, v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def resize(self, slots, lens):
        B.pages_resize(self.book, self.page_pools, self.ints(slots), self.ints(lens), len(slots), self.result, self.scratch, self.need,
                       torch.cuda.current_stream())
        assert self.want.resize(slots, lens)[0] == self.result.item() == 0
        for s, n in zip(slots, lens):
            for layer in range(LAYERS):
                self.keys[s][layer], self.values[s][layer] = self.keys[s][layer][:n], self.values[s][layer][:n]
            self.tokens[s] = self.tokens[s][:n]

    def fork(self, src, dst):
        B.pages_fork(self.book, self.ints(src), self.ints(dst), len(src), self.scratch, self.need, torch.cuda.current_stream())
        self.want.fork(src, dst)
        old = [(list(k), list(v), list(t)) for k, v, t in zip(self.keys, self.values, self.tokens)]
        for a, b in zip(src, dst):
            self.keys[b], self.values[b], self.tokens[b] = (list(x) for x in old[a])

    def compact(self):
        B.pages_compact(self.book, self.page_pools, self.result, self.scratch, self.need, torch.cuda.current_stream())
        assert self.want.compact()[0] == self.result.item()

    def same_book(self):
        return (self.book.refs.tolist() == self.want.refs and self.book.lens.tolist() == self.want.lens
                and self.book.table.tolist() == self.want.table and self.want.consistent())

    def forward(self, slots, tokens):
        """tokens[i]: the new tokens of the sequence in slot slots[i], for which there is room; returns logits (items, longest, vocab)."""
        n, longest = len(slots), max(len(t) for t in tokens)
        news, slot_of = self.ints([len(t) for t in tokens]), self.ints(slots)
        ids = torch.tensor([t + [0] * (longest - len(t)) for t in tokens], device="cuda")
        x = self.embed[ids].view(n * longest, DIM)
        for layer in range(LAYERS):
            qkv = product(x, self.wqkv[layer]).view(n, longest, HQ + 2 * HK, HEAD)
            q, k_new, v_new = qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HK], qkv[:, :, HQ + HK:]
            k, v = self.pools[layer][:, 0], self.pools[layer][:, 1]
            o = torch.zeros(n, longest, HQ, HEAD, dtype=BF, device="cuda")
            shape = B.PagedShape.of(q, k, v, o, self.book.table, k_new, v_new)
            B.cache_append(shape, k_new, v_new, k, v, self.book.table, self.book.lens, slot_of, news, torch.cuda.current_stream())
            size = B.paged_attn_scratch_bytes(shape)
            scratch = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
            B.paged_attn(shape, q, k, v, self.book.table, self.book.lens, slot_of, news, o, None, scratch, size, torch.cuda.current_stream())
            for i, s in enumerate(slots):
                m = len(tokens[i])
                self.keys[s][layer] = torch.cat([self.keys[s][layer], k_new[i, :m]])
                self.values[s][layer] = torch.cat([self.values[s][layer], v_new[i, :m]])
                self.check(q[i, :m], o[i, :m], self.keys[s][layer], self.values[s][layer])
                assert not o[i, m:].any()
            x = (x.float() + product(o.view(n * longest, -1), self.wo[layer]).float()).to(BF)
        for s, t in zip(slots, tokens):
            self.tokens[s] = self.tokens[s] + t
        return product(x, self.embed.t(), True).view(n, longest, VOCAB) * 0.02

    @staticmethod
    def check(q, o, k, v):
        m, length = len(q), len(k)
        kh, vh = (t.double().transpose(0, 1).repeat_interleave(HQ // HK, 0) for t in (k, v))
        z = q.double().transpose(0, 1) @ kh.transpose(1, 2) * HEAD ** -0.5
        hidden = torch.arange(length, device="cuda") > length - m + torch.arange(m, device="cuda")[:, None]
        want = (torch.softmax(z.masked_fill(hidden, float("-inf")), 2) @ vh).transpose(0, 1)
        assert bool(((o.double() - want).abs() <= 2.1 * H * (want.abs() + vh.abs().max())).all())


def answer_step(s, slots, seed):
    """Drafts behind each sequence's last token, checked by the target, what is not accepted given back; the number accepted."""
    n = len(slots)
    g = torch.Generator(device="cuda").manual_seed(seed)
    had = [len(s.tokens[i]) for i in slots]
    q = torch.softmax(torch.randn(n, DRAFTS, VOCAB, generator=g, device="cuda"), 2)
    drafts = torch.multinomial(q.view(n * DRAFTS, VOCAB), 1, generator=g).view(n, DRAFTS).int()
    lens = torch.randint(0, DRAFTS + 1, (n,), generator=g, device="cuda").int()
    last = s.pending
    s.resize(slots, [h + 1 + m for h, m in zip(had, lens.tolist())])
    logits = s.forward(slots, [[last[i]] + drafts[j, :m].tolist() for j, (i, m) in enumerate(zip(slots, lens.tolist()))])
    p = torch.full((n, DRAFTS + 1, VOCAB), float("nan"), device="cuda")
    p[:, :logits.shape[1]] = torch.softmax(logits, 2)
    u = torch.rand(n, DRAFTS + 1, generator=g, device="cuda")
    tokens, accepted = torch.empty(n, DRAFTS + 1, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    B.draft_verify(p, q, drafts, lens, u, tokens, accepted, n, DRAFTS, VOCAB, VOCAB, VOCAB, B.F32, torch.cuda.current_stream())
    for j, (i, m, a) in enumerate(zip(slots, lens.tolist(), accepted.tolist())):
        want = 0
        while want < m and float(u[j, want]) * float(q[j, want, drafts[j, want]]) < float(p[j, want, drafts[j, want]]):
            want += 1
        assert a == want and tokens[j, :a].tolist() == drafts[j, :a].tolist() and tokens[j, a + 1:].tolist() == [-1] * (DRAFTS - a)
        last[i] = tokens[j, a].item()
        assert 0 <= last[i] < VOCAB
    s.resize(slots, [h + 1 + a for h, a in zip(had, accepted.tolist())])
    return accepted.sum().item()


def test_answering_with_drafts():
    s = Server(6, 120, 12)
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(0, VOCAB, (n,), generator=g).tolist() for n in (1, 17, 8, 30)]
    slots = [4, 0, 3, 1]
    s.resize(slots, [len(p) for p in prompts])
    logits = s.forward(slots, prompts)
    s.pending = {i: int(logits[j, len(p) - 1].argmax()) for j, (i, p) in enumerate(zip(slots, prompts))}
    got = 0
    for step in range(8):
        got += answer_step(s, slots, step)
        if step == 2:
            s.compact()
        if step == 4:
            s.fork([0, 0], [2, 5])                     # two more continuations of one sequence
            s.pending.update({2: 11, 5: 12})
            slots = slots + [2, 5]
        if step == 6:
            s.resize([3, 4], [0, 0])                   # two end
            slots = [i for i in slots if i not in (3, 4)]
            s.compact()
        assert s.same_book()
    assert got > 0
    s.resize(slots, [0] * len(slots))
    assert s.same_book() and not any(s.want.refs)


def test_a_fork_answers_like_its_own_prompt_and_pages_may_move():
    """A continuation of a forked sequence, of one whose prompt was written by itself, and of the same after the pages
    have moved: the same bits."""
    g = torch.Generator().manual_seed(9)
    prompt, more = (torch.randint(0, VOCAB, (n,), generator=g).tolist() for n in (21, 5))
    outs = []
    for way in ("alone", "fork", "moved"):
        s = Server(3, 40, 8, seed=2)
        if way == "moved":
            s.resize([2], [30])
        s.resize([0], [len(prompt)])
        s.forward([0], [prompt])
        slot = 0
        if way == "fork":
            s.fork([0], [1])
            s.resize([0], [len(prompt) + 1])
            s.forward([0], [[7]])                      # the parent goes on by itself
            slot = 1
        if way == "moved":
            s.resize([2], [0])
            s.compact()
        s.resize([slot], [len(prompt) + len(more)])
        outs.append(s.forward([slot], [more]))
        assert s.same_book()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_a_step_as_a_graph():
    """Resize, append, attend and verify captured once and replayed while the sequences grow on the device."""
    n, steps = 4, 12
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    book = B.PageBook(60, 4, n, 12)
    pool = torch.full((60, 2, 4, HK, HEAD), float("nan"), dtype=BF, device="cuda")
    pools = B.page_pools([pool])
    need = B.pages_resize_scratch_bytes(book, n)
    scratch, result = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    want = torch.tensor([3, 9, 1, 12], dtype=torch.int32, device="cuda")
    qkv = torch.empty(n, 1, HQ + 2 * HK, HEAD, dtype=BF, device="cuda")
    q, k_new, v_new = qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HK], qkv[:, :, HQ + HK:]
    o, u = torch.empty(n, 1, HQ, HEAD, dtype=BF, device="cuda"), torch.empty(n, 1, device="cuda")
    p = torch.empty(n, 1, VOCAB, device="cuda")
    tokens, accepted = torch.empty(n, 1, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    drafts = torch.empty(n, 0, dtype=torch.int32, device="cuda")
    shape = B.PagedShape.of(q, pool[:, 0], pool[:, 1], o, book.table, k_new, v_new)
    size = B.paged_attn_scratch_bytes(shape)
    att = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream()
    B.pages_resize(book, pools, None, want, n, result, scratch, need, s)
    keys, values = [rnd(m, HK, HEAD).to(BF) for m in want.tolist()], [rnd(m, HK, HEAD).to(BF) for m in want.tolist()]
    for i in range(n):                                 # what is there so far
        at = torch.arange(len(keys[i]), device="cuda")
        pool[book.table[i].long()[at // 4], 0, at % 4], pool[book.table[i].long()[at // 4], 1, at % 4] = keys[i], values[i]

    def step():
        s = torch.cuda.current_stream()
        want.add_(1)
        B.pages_resize(book, pools, None, want, n, result, scratch, need, s)
        B.cache_append(shape, k_new, v_new, pool[:, 0], pool[:, 1], book.table, book.lens, None, None, s)
        B.paged_attn(shape, q, pool[:, 0], pool[:, 1], book.table, book.lens, None, None, o, None, att, size, s)
        B.draft_verify(p, None, drafts, None, u, tokens, accepted, n, 0, VOCAB, VOCAB, VOCAB, B.F32, s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(steps):
        qkv.copy_(rnd(n, 1, HQ + 2 * HK, HEAD))
        p.copy_(torch.softmax(rnd(n, 1, VOCAB), 2))
        u.uniform_(generator=gen)
        graph.replay()
        assert result.item() == 0 and book.lens.tolist() == want.tolist()
        sums = p.double().cumsum(2)
        assert tokens.flatten().tolist() == [int((sums[i, 0] <= u[i, 0].double() * sums[i, 0, -1]).sum()) for i in range(n)]
        for i in range(n):
            keys[i], values[i] = torch.cat([keys[i], k_new[i]]), torch.cat([values[i], v_new[i]])
            Server.check(q[i], o[i], keys[i], values[i])


@pytest.mark.parametrize("task,size", [("paged-attn", 300), ("paged-drafts", 300), ("cache-append", 20), ("pages-copy", 3), ("draft-verify", 999)])
def test_harness_cache_commands_run(task, size, capsys):
    import json
    from paper_2506_09092_b200 import harness as H
    H._main(["--task", task, "--size", str(size), "--iters", "2", "--warmup", "1"])
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["task"] == task and line["status"] == 0 and line["us_median"] > 0
