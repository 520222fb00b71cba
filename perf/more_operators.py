"""Workloads for timing the operators of answering from a paged cache: attention of the newest tokens over
the pages, appending keys and values, forking / resizing sequences and compacting the pages, and the
verification of drafted tokens.

``own`` False computes a case from elementary torch operations; ``own`` True calls the library's entry
points.  Both take what ``prepare`` returns.
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
_CODES = {"fp32": 0, "bf16": 1, "fp16": 2}


# ------------------------------------------------------------------ cases --
def listed():
    return [
        # one sequence, one token, a short answer so far: latency counts
        dict(name="attn_one", op="attn", batch=1, rows=1, heads=8, kv_heads=8, dim=64, length=300, page_rows=16,
             dtype="fp16", layout="rows", ragged=False, slots=False, lse=False),
        # a batch of sequences of all lengths, each one token further
        dict(name="attn_batch", op="attn", batch=48, rows=1, heads=32, kv_heads=8, dim=128, length=4096, page_rows=16,
             dtype="bf16", layout="rows", ragged=True, slots=True, lse=False),
        # up to four drafted tokens and the one before them, checked together
        dict(name="attn_drafts", op="attn", batch=16, rows=5, heads=32, kv_heads=4, dim=128, length=8192, page_rows=64,
             dtype="fp16", layout="heads", ragged=True, slots=False, lse=True),
        # two very long documents
        dict(name="attn_long", op="attn", batch=2, rows=1, heads=64, kv_heads=8, dim=128, length=131072, page_rows=128,
             dtype="bf16", layout="joint", ragged=False, slots=False, lse=False),
        # a token's keys and values of eight sequences
        dict(name="append_token", op="append", batch=8, rows=1, heads=32, kv_heads=8, dim=128, length=1000, page_rows=16,
             dtype="bf16", layout="rows", ragged=False, slots=False),
        # four prompts, written at once
        dict(name="append_prompt", op="append", batch=4, rows=2048, heads=32, kv_heads=8, dim=128, length=2600, page_rows=16,
             dtype="bf16", layout="rows", ragged=True, slots=True),
        # four sequences, a toy vocabulary
        dict(name="verify_small", op="verify", batch=4, drafts=3, vocab=1000, dtype="fp32", certain=False, ragged=True),
        # sixty-four sequences with five drafts each over a large vocabulary
        dict(name="verify_large", op="verify", batch=64, drafts=5, vocab=128000, dtype="fp32", certain=False, ragged=False),
        # a step of a small beam search: two groups of four continue from their parents
        dict(name="beam_small", op="beam", groups=2, beams=4, prompt_pages=3, own_pages=2, page_rows=16, layers=2, width=512,
             grow=1),
        # 32 groups of eight, sixteen layers
        dict(name="beam_large", op="beam", groups=32, beams=8, prompt_pages=8, own_pages=3, page_rows=16, layers=16, width=1024,
             grow=1),
        # a small pool after some sequences have ended
        dict(name="compact_small", op="compact", slots=16, pages=200, live=0.5, page_rows=16, layers=2, width=512),
        # a pool of eight layers, somewhat more than half in use
        dict(name="compact_large", op="compact", slots=100, pages=3001, live=0.55, page_rows=16, layers=8, width=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "append", "verify", "beam", "compact"])
    if op == "verify":
        vocab, drafts, batch = _log_int(rng, 50, 200000), rng.randint(1, 8), _log_int(rng, 1, 128)
        while batch * (drafts + 1) * vocab > 48000000:
            batch //= 2
        return dict(op=op, batch=batch, drafts=drafts, vocab=vocab, dtype=rng.choice(["fp32", "fp32", "bf16", "fp16"]),
                    certain=rng.random() < 0.25, ragged=rng.random() < 0.5)
    if op == "beam":
        groups, beams, layers, width = _log_int(rng, 1, 32), rng.randint(1, 8), rng.randint(1, 16), 8 * _log_int(rng, 4, 128)
        return dict(op=op, groups=groups, beams=beams, prompt_pages=rng.randint(0, 8), own_pages=rng.randint(1, 3),
                    page_rows=rng.choice([1, 5, 8, 16]), layers=layers, width=width, grow=rng.choice([1, 1, 2, 7]))
    if op == "compact":
        pages = _log_int(rng, 10, 3000)
        return dict(op=op, slots=rng.randint(1, 120), pages=pages, live=round(rng.uniform(0.1, 0.95), 2),
                    page_rows=rng.choice([1, 8, 16]), layers=rng.randint(1, 8), width=8 * _log_int(rng, 4, 128))
    kv_heads, dim = rng.choice([1, 2, 4, 8, 16]), rng.choice([32, 64, 80, 96, 128, 128])
    group = rng.choice([1, 2, 4, 8]) if kv_heads <= 8 else 1
    case = dict(op=op, batch=_log_int(rng, 1, 64), rows=rng.choice([1, 1, 1, 2, 3, 4, 6, 8]), heads=kv_heads * group,
                kv_heads=kv_heads, dim=dim, length=0, page_rows=rng.choice([1, 8, 16, 16, 24, 32, 64, 100, 128, 256]),
                dtype=rng.choice(["bf16", "fp16"]), layout=rng.choice(["rows", "heads", "joint"]),
                ragged=rng.random() < 0.6, slots=rng.random() < 0.5)
    if op == "append":
        case["rows"] = _log_int(rng, 1, 2048)
        case["length"] = case["rows"] + _log_int(rng, 1, 2000)
        while case["batch"] * case["length"] * kv_heads * dim > (1 << 24) and case["batch"] > 1:
            case["batch"] //= 2
        return case
    case["lse"] = rng.random() < 0.5
    case["length"] = case["rows"] + _log_int(rng, 1, 100000)
    while case["batch"] * case["length"] * kv_heads * dim > (1 << 27):
        case["length"] = max(case["rows"], case["length"] // 2)
    return case


# ------------------------------------------- what a case's numbers stand for --
def _lens(case):
    """States of each sequence, the new ones among them: all of them, or from a quarter on."""
    b, n, t = case["batch"], case["length"], case["rows"]
    return [max(t, n - (i * n * 3) // (4 * b)) if case["ragged"] else n for i in range(b)]


def _news(case):
    """New tokens of each sequence."""
    t = case["rows"]
    return [1 + (5 * i + t - 1) % t if case["ragged"] else t for i in range(case["batch"])]


def _draft_lens(case):
    t = case["drafts"]
    return [1 + (3 * i + t - 1) % t if case["ragged"] else t for i in range(case["batch"])]


def _cdiv(a, b):
    return (a + b - 1) // b


def _beam_book(case):
    """(refs, lens, table, parents): groups of sequences that share a prompt's pages and have pages of their own behind
    it; the parents that the next step's sequences continue from."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    g, k, r = case["groups"], case["beams"], case["page_rows"]
    pages = g * (case["prompt_pages"] + 2 * k * (case["own_pages"] + _cdiv(case["grow"], r) + 1))
    cols = case["prompt_pages"] + case["own_pages"] + _cdiv(case["grow"], r) + 2
    ids = list(range(pages))
    rng.shuffle(ids)
    refs, lens, table, parents = [0] * pages, [], [], []
    for i in range(g):
        prompt = [ids.pop() for _ in range(case["prompt_pages"])]
        for p in prompt:
            refs[p] = k
        last = rng.randint(1, r)                       # of the beams' own pages: they all are as long
        for _ in range(k):
            mine = [ids.pop() for _ in range(case["own_pages"])]
            for p in mine:
                refs[p] = 1
            table.append(prompt + mine + [-1] * (cols - len(prompt) - len(mine)))
            lens.append((len(prompt) + len(mine) - 1) * r + last)
            parents.append(i * k + rng.randrange(k))
    return refs, lens, table, parents


def _beam_copies(case):
    """Pages that the step copies: of the beams of one parent all but the first, where the last page is not full."""
    refs, lens, table, parents = _beam_book(case)
    return sum(1 for i, p in enumerate(parents) if lens[p] % case["page_rows"] and p in parents[:i])


def _compact_book(case):
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    pages, r, slots = case["pages"], case["page_rows"], case["slots"]
    ids = rng.sample(range(pages), max(1, int(pages * case["live"])))
    cuts = sorted(rng.randint(0, len(ids)) for _ in range(slots - 1))
    spans = list(zip([0] + cuts, cuts + [len(ids)]))
    cols = max(b - a for a, b in spans) + 1
    refs, lens, table = [0] * pages, [], []
    for i, (a, b) in enumerate(spans):
        mine = ids[a:b]
        if i % 5 == 4 and i and table[i - 1][0] >= 0:  # a sequence that shares its first page with its neighbour
            mine = [table[i - 1][0]] + mine[1:] if mine else mine
        for p in mine:
            refs[p] += 1
        lens.append(max(0, len(mine) * r - rng.randrange(r)))
        table.append(mine + [-1] * (cols - len(mine)))
    return refs, lens, table


def _compact_moves(case):
    refs = _compact_book(case)[0]
    live = sum(1 for n in refs if n)
    return sum(1 for p in range(live, len(refs)) if refs[p])


def work(case):
    op = case["op"]
    if op in ("attn", "append"):
        es, d, hk = _BYTES[case["dtype"]], case["dim"], case["kv_heads"]
        lens, news = _lens(case), _news(case)
        if op == "append":
            return {"bytes": 4 * sum(news) * hk * d * es, "flops": 0}
        q_values = sum(news) * case["heads"] * d
        pairs = sum(n * (2 * l - n + 1) // 2 for l, n in zip(lens, news)) * case["heads"]
        table = 4 * sum(_cdiv(l, case["page_rows"]) for l in lens)
        lse = 4 * sum(news) * case["heads"] if case["lse"] else 0
        return {"bytes": 2 * sum(lens) * hk * d * es + 2 * q_values * es + table + lse, "flops": 4 * pairs * d}
    if op == "verify":
        rows = case["batch"] * (1 if case["certain"] else 2)
        return {"bytes": rows * case["vocab"] * _BYTES[case["dtype"]], "flops": 2 * rows * case["vocab"]}
    page = 2 * case["layers"] * case["page_rows"] * case["width"] * 2
    if op == "beam":
        refs, lens, table, _ = _beam_book(case)
        used = sum(_cdiv(n, case["page_rows"]) for n in lens)
        return {"bytes": 2 * page * _beam_copies(case) + 4 * (2 * used + 4 * len(lens)), "flops": 0}
    refs, lens, table = _compact_book(case)
    return {"bytes": 2 * page * _compact_moves(case) + 4 * (2 * len(refs) + 2 * sum(_cdiv(n, case["page_rows"]) for n in lens)),
            "flops": 0}


# ----------------------------------------------------------------- inputs --
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cache_inputs(case, gen):
    """Pages in use by the sequences in a random order, the rest of the pool holding something else."""
    t, b, r, hk, d = _TYPES[case["dtype"]], case["batch"], case["page_rows"], case["kv_heads"], case["dim"]
    lens, news = _lens(case), _news(case)
    counts = [_cdiv(n, r) for n in lens]
    pages, cols = sum(counts) + 1 + sum(counts) // 16, max(counts) + 3
    slots = b + 5 if case["slots"] else b
    order = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int32)
    s = dict(lens_host=lens, news_host=news)
    where = list(range(b))
    if case["slots"]:
        where = torch.randperm(slots, generator=gen, device="cuda")[:b].tolist()
        s["slots"] = _ints(where)
    else:
        s["slots"] = None
    table, all_lens, at = torch.full((slots, cols), -1, dtype=torch.int32, device="cuda"), [0] * slots, 0
    for i, w in enumerate(where):
        table[w, :counts[i]] = order[at:at + counts[i]]
        all_lens[w] = lens[i]
        at += counts[i]
    s["table"], s["lens"] = table, _ints(all_lens)
    s["news"] = _ints(news) if case["ragged"] else None
    s["where"] = where

    def values(*shape):
        out = torch.empty(*shape, dtype=t, device="cuda")
        return out.normal_(generator=gen)
    if case["layout"] == "joint":                      # keys and values of a page side by side
        pool = values(pages, 2, r, hk, d)
        s["pools"], s["k"], s["v"] = [pool], pool[:, 0], pool[:, 1]
    elif case["layout"] == "heads":                    # the rows of a head together
        s["pools"] = [values(pages, hk, r, d) for _ in range(2)]
        s["k"], s["v"] = (p.transpose(1, 2) for p in s["pools"])
    else:
        s["pools"] = [values(pages, r, hk, d) for _ in range(2)]
        s["k"], s["v"] = s["pools"]
    # queries, keys and values of the new tokens as one projection writes them
    hq = case["heads"]
    qkv = values(b, case["rows"], hq + 2 * hk, d)
    s["q"], s["k_new"], s["v_new"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:]
    return s


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 6007 + 29)
    op = case["op"]
    if op in ("attn", "append"):
        return _cache_inputs(case, gen)
    if op == "verify":
        b, n, v, t = case["batch"], case["drafts"], case["vocab"], _TYPES[case["dtype"]]
        logits = torch.randn(b, n + 1, v, generator=gen, device="cuda").mul_(2.5)
        p = torch.softmax(logits, 2)
        u = torch.rand(b, n + 1, generator=gen, device="cuda")
        s = dict(p=p.to(t), u=u, q=None, draft_lens=_ints(_draft_lens(case)) if case["ragged"] else None)
        if case["certain"]:                            # drafts looked up in the text so far: no distribution of their own
            s["drafts"] = torch.multinomial(p[:, :n].reshape(b * n, v), 1, generator=gen).view(b, n).int()
        else:
            q = torch.softmax(logits[:, :n] + torch.randn(b, n, v, generator=gen, device="cuda").mul_(0.7), 2)
            s["q"] = q.to(t)
            s["drafts"] = torch.multinomial(q.reshape(b * n, v), 1, generator=gen).view(b, n).int()
        return s
    if op == "beam":
        refs, lens, table, parents = _beam_book(case)
        s = dict(parents=_ints(parents), slots=torch.arange(len(lens), dtype=torch.int32, device="cuda"),
                 want=_ints([lens[p] + case["grow"] for p in parents]))
    else:
        refs, lens, table = _compact_book(case)
        s = {}
    s["start"] = torch.cat([_ints(refs), _ints(lens), _ints(table).flatten()])
    s["sizes"] = (len(refs), len(lens), len(table[0]))
    # keys and values of every layer
    s["pool"] = torch.empty(2 * case["layers"], len(refs), case["page_rows"] * case["width"], dtype=torch.bfloat16,
                            device="cuda").normal_(generator=gen)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if op == "attn":
        b, t, hq, d = case["batch"], case["rows"], case["heads"], case["dim"]
        s["out"] = torch.zeros(b, t, hq, d, dtype=_TYPES[case["dtype"]], device="cuda")
        s["out_lse"] = torch.zeros(b, hq, t, device="cuda") if case["lse"] else None
    elif op == "verify":
        s["tokens"] = torch.empty(case["batch"], case["drafts"] + 1, dtype=torch.int32, device="cuda")
        s["accepted"] = torch.empty(case["batch"], dtype=torch.int32, device="cuda")
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a user's program sets up once: sizes and strides, the book of pages, tables of pools, scratch."""
    from paper_2506_09092_b200 import binding as lib
    case = s["case"]
    op = case["op"]
    s["lib"] = lib
    need = 0
    if op in ("attn", "append"):
        s["shape"] = lib.PagedShape.of(s["q"], s["k"], s["v"], s.get("out", s["q"]), s["table"], s["k_new"], s["v_new"])
        if op == "attn":
            need = lib.paged_attn_scratch_bytes(s["shape"])
    elif op in ("beam", "compact"):
        pages, slots, cols = s["sizes"]
        book = lib.PageBook(pages, case["page_rows"], slots, cols)
        n = pages + slots
        book.refs.copy_(s["start"][:pages])
        book.lens.copy_(s["start"][pages:n])
        book.table.copy_(s["start"][n:].view(slots, cols))
        s["book"], s["book_start"] = book, book.data.clone()
        s["page_pools"] = lib.page_pools(list(s["pool"]))
        s["result"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if op == "beam":
            need = max(lib.pages_fork_scratch_bytes(book, slots), lib.pages_resize_scratch_bytes(book, slots))
        else:
            need = lib.pages_compact_scratch_bytes(book)
    s["scratch"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    s["need"] = need


# ------------------------------------------------------------------- runs --
def run(s):
    if own:
        return _run_own(s)
    return _PLAIN[s["case"]["op"]](s)


def _run_own(s):
    if "lib" not in s:
        _plan(s)
    lib, case = s["lib"], s["case"]
    op, stream = case["op"], torch.cuda.current_stream()
    if op == "attn":
        lib.paged_attn(s["shape"], s["q"], s["k"], s["v"], s["table"], s["lens"], s["slots"], s["news"], s["out"],
                       s["out_lse"], s["scratch"], s["need"], stream)
        return s["out"] if s["out_lse"] is None else (s["out"], s["out_lse"])
    if op == "append":
        lib.cache_append(s["shape"], s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["lens"], s["slots"], s["news"],
                         stream)
        return s["pools"]
    if op == "verify":
        v = case["vocab"]
        lib.draft_verify(s["p"], s["q"], s["drafts"], s["draft_lens"], s["u"], s["tokens"], s["accepted"], case["batch"],
                         case["drafts"], v, v, v, _CODES[case["dtype"]], stream)
        return s["tokens"], s["accepted"]
    book = s["book"]
    book.data.copy_(s["book_start"])                   # the same step again
    if op == "beam":
        n = len(s["slots"])
        lib.pages_fork(book, s["parents"], s["slots"], n, s["scratch"], s["need"], stream)
        lib.pages_resize(book, s["page_pools"], s["slots"], s["want"], n, s["result"], s["scratch"], s["need"], stream)
    else:
        lib.pages_compact(book, s["page_pools"], s["result"], s["scratch"], s["need"], stream)
    return s["result"], book.refs, book.lens, book.table, s["pool"]


def _rows_of(s):
    """Table rows and lengths of the batch's sequences, their new tokens."""
    case = s["case"]
    table, lens = s["table"], s["lens"]
    if s["slots"] is not None:
        table, lens = table[s["slots"]], lens[s["slots"]]
    news = s["news"] if s["news"] is not None else torch.full_like(lens, case["rows"])
    return table, lens, news


def _attn(s):
    case = s["case"]
    b, t, hq, hk, d, r = (case[k] for k in ("batch", "rows", "heads", "kv_heads", "dim", "page_rows"))
    table, lens, news = _rows_of(s)
    top = max(s["lens_host"])
    ids = table[:, :_cdiv(top, r)].clamp(min=0)
    k = s["k"][ids].reshape(b, -1, hk, d)[:, :top].float().transpose(1, 2)        # batch, key head, states, dim
    v = s["v"][ids].reshape(b, -1, hk, d)[:, :top].float().transpose(1, 2)
    q = s["q"].float().view(b, t, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    z = torch.matmul(q, k.transpose(2, 3)).mul_(d ** -0.5).view(b, hk, hq // hk, t, top)
    at = (lens - news)[:, None] + torch.arange(t, device="cuda")               # position of each query
    hidden = torch.arange(top, device="cuda") > at[:, :, None]
    z = z.masked_fill_(hidden[:, None, None], float("-inf"))
    m = z.amax(4, keepdim=True)
    p = z.sub_(m).exp_()
    total = p.sum(4, keepdim=True)
    o = torch.matmul(p.view(b, hk, -1, top), v).view(b, hk, hq // hk, t, d) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(b, t, hq, d)
    there = torch.arange(t, device="cuda") < news[:, None]
    o = torch.where(there[:, :, None, None], o, 0.0).to(s["q"].dtype)
    if not case["lse"]:
        return o
    return o, torch.where(there[:, None], (m + total.log()).squeeze(4).reshape(b, hq, t), 0.0)


def _append(s):
    case = s["case"]
    t, r = case["rows"], case["page_rows"]
    table, lens, news = _rows_of(s)
    item = torch.arange(case["batch"], device="cuda")[:, None]
    new = torch.minimum(torch.arange(t, device="cuda"), news[:, None] - 1)     # rows behind the last: the last again
    at = (lens - news)[:, None] + new
    page = table.gather(1, (at // r).long())
    s["k"][page, at % r] = s["k_new"][item, new]
    s["v"][page, at % r] = s["v_new"][item, new]
    return s["pools"]


def _verify(s):
    case = s["case"]
    b, n = case["batch"], case["drafts"]
    p, x = s["p"], s["drafts"].long()
    count = s["draft_lens"].long() if s["draft_lens"] is not None else torch.full((b,), n, device="cuda")
    px = p[:, :n].gather(2, x[:, :, None]).squeeze(2).double()
    qx = torch.ones_like(px) if s["q"] is None else s["q"].gather(2, x[:, :, None]).squeeze(2).double()
    steps = torch.arange(n, device="cuda")
    good = (s["u"][:, :n].double() * qx < px) & (steps < count[:, None])
    accepted = good.long().cumprod(1).sum(1)
    item = torch.arange(b, device="cuda")
    row = p[item, accepted].double()
    last = accepted.clamp(max=n - 1)
    if s["q"] is None:
        other = torch.zeros_like(row).scatter_(1, x[item, last][:, None], 1.0)
    else:
        other = s["q"][item, last].double()
    mass = torch.where((accepted < count)[:, None], (row - other).clamp(min=0), row)
    total = mass.sum(1, keepdim=True)
    mass = torch.where(total > 0, mass, row)
    sums = mass.cumsum(1)
    hit = (sums > s["u"][:, n:].double() * sums[:, -1:]) & (mass > 0)
    token = hit.int().argmax(1)
    cols = torch.arange(n + 1, device="cuda")
    tokens = torch.where(cols < accepted[:, None], torch.nn.functional.pad(x, (0, 1)), -1)
    tokens = torch.where(cols == accepted[:, None], token[:, None], tokens)
    return tokens.int(), accepted.int()


def _parts(s):
    pages, slots, cols = s["sizes"]
    flat = s["start"].clone()
    return flat[:pages], flat[pages:pages + slots], flat[pages + slots:].view(slots, cols)


def _beam(s):
    case = s["case"]
    r, grow, pool = case["page_rows"], case["grow"], s["pool"]
    refs, lens, table = _parts(s)
    pages, cols = len(refs), torch.arange(table.shape[1], device="cuda")
    src, dst = s["parents"].long(), s["slots"].long()
    # every sequence becomes its parent
    old_there, new_there = cols < ((lens[dst] + r - 1) // r)[:, None], cols < ((lens[src] + r - 1) // r)[:, None]
    old_ids, new_ids = table[dst], table[src]
    refs.index_add_(0, new_ids.clamp(min=0).flatten(), new_there.int().flatten())
    refs.index_add_(0, old_ids.clamp(min=0).flatten(), -old_there.int().flatten())
    table[dst] = torch.where(new_there, new_ids, old_ids)
    lens[dst] = lens[src]
    # and longer: shared last pages are exchanged for copies, new pages taken from the lowest free ones
    old, new = lens[dst], s["want"]
    old_pages, new_pages = (old + r - 1) // r, (new + r - 1) // r
    tail_at = (old_pages - 1).clamp(min=0).long()
    tail = table[dst, tail_at].long()
    shared = (new > old) & (old % r != 0) & (refs[tail] > 1)
    claims = torch.zeros_like(refs).index_add_(0, tail, shared.int())
    index = torch.arange(len(dst), device="cuda", dtype=torch.int32)
    first = torch.full_like(refs, len(dst)).scatter_reduce_(0, tail, torch.where(shared, index, len(dst)), "amin")
    copied = shared & ~((claims[tail] == refs[tail]) & (first[tail] == index))
    need = new_pages - old_pages + copied
    start = (need.cumsum(0) - need).long()
    free = torch.argsort((refs > 0).int(), stable=True)
    fresh = free[start]
    refs.index_add_(0, tail, -copied.int())
    pool[:, torch.where(copied, fresh, tail)] = pool[:, tail]
    table[dst, tail_at] = torch.where(copied, fresh, tail).int()
    refs.index_add_(0, fresh, copied.int())
    for i in range(_cdiv(grow, r)):
        more = old_pages + i < new_pages
        at = (old_pages + i).clamp(max=table.shape[1] - 1).long()
        page = free[(start + copied + i).clamp(max=pages - 1)]
        table[dst, at] = torch.where(more, page.int(), table[dst, at])
        refs.index_add_(0, page, more.int())
    lens[dst] = new
    return torch.zeros(1, dtype=torch.int32, device="cuda"), refs, lens, table, pool


def _compact(s):
    r, pool = s["case"]["page_rows"], s["pool"]
    refs, lens, table = _parts(s)
    live = refs > 0
    used = live.sum().int().view(1)
    ids = torch.arange(len(refs), device="cuda", dtype=torch.int32)
    movers, holes = (live & (ids >= used)).nonzero()[:, 0], (~live & (ids < used)).nonzero()[:, 0]
    ids[movers] = holes.int()
    pool[:, holes] = pool[:, movers]
    refs[holes] = refs[movers]
    refs[movers] = 0
    there = torch.arange(table.shape[1], device="cuda") < ((lens + r - 1) // r)[:, None]
    return used, refs, lens, torch.where(there, ids[table.clamp(min=0)], table), pool


_PLAIN = dict(attn=_attn, append=_append, verify=_verify, beam=_beam, compact=_compact)


# ------------------------------------------------------------------ exact --
def exact(case, seed):
    """Attention in 64 bits, one sequence and key head at a time; tokens by the definition, one sequence at a time.
    The other operators move values and count pages: nothing is computed."""
    op = case["op"]
    if op not in ("attn", "verify"):
        return None
    s = _inputs(case, seed)
    if op == "verify":
        tokens, counts = [], []
        b, n = case["batch"], case["drafts"]
        u, x = s["u"].double().tolist(), s["drafts"].tolist()
        for i, count in enumerate(_draft_lens(case)):
            a = 0
            while a < count:
                p = float(s["p"][i, a, x[i][a]])
                q = 1.0 if s["q"] is None else float(s["q"][i, a, x[i][a]])
                if not u[i][a] * q < p:
                    break
                a += 1
            mass = s["p"][i, a].double()
            if a < count:
                if s["q"] is None:
                    rest = mass.clone()
                    rest[x[i][a]] = max(0.0, float(rest[x[i][a]]) - 1.0)
                else:
                    rest = torch.relu(mass - s["q"][i, a].double())
                mass = rest if float(rest.sum()) > 0 else mass
            sums = torch.cumsum(mass, 0)
            token = int(torch.searchsorted(sums, u[i][n] * sums[-1:], right=True))
            tokens.append(x[i][:a] + [token] + [-1] * (n - a))
            counts.append(a)
        return _ints(tokens), _ints(counts)
    t, hq, hk, d, r = (case[k] for k in ("rows", "heads", "kv_heads", "dim", "page_rows"))
    g = hq // hk
    out = torch.zeros(case["batch"], t, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(case["batch"], hq, t, dtype=torch.float64, device="cuda")
    for i, (length, n) in enumerate(zip(_lens(case), _news(case))):
        ids = s["table"][s["where"][i], :_cdiv(length, r)].long()
        keep = torch.ones(n, length, dtype=torch.bool, device="cuda").tril(length - n)
        for h in range(hk):
            k = s["k"][ids, :, h].reshape(-1, d)[:length].double()
            v = s["v"][ids, :, h].reshape(-1, d)[:length].double()
            for j in range(h * g, h * g + g):
                z = (s["q"][i, :n, j].double() @ k.T) / math.sqrt(d)
                z[~keep] = -math.inf
                lse[i, j, :n] = torch.logsumexp(z, 1)
                out[i, :n, j] = torch.softmax(z, 1) @ v
    return (out, lse) if case["lse"] else out
