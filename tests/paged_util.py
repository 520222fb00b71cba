"""A paged cache for tests: random pages in some layout, everything outside the sequences' own rows poisoned, and the
attention of the newest tokens over it in 64 bits."""
import torch

from paper_2506_09092_b200 import binding as B

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def cdiv(a, b):
    return (a + b - 1) // b


class Cache:
    """``lens[b]`` states of item b (new tokens among them) in slot ``where[b]``; the rows of the pools that no sequence
    has hold NaN and infinities."""

    def __init__(self, lens, rows, hq, hk, dim, dtype="bf16", page_rows=16, layout="rows", slots=None, news=None, cols=None,
                 spread=1.5, seed=0, spare=3, poison=True):
        t, b = TYPES[dtype], len(lens)
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.lens_host, self.rows, self.news_host = list(lens), rows, [rows] * b if news is None else list(news)
        self.dtype, self.page_rows, self.hq, self.hk, self.dim = dtype, page_rows, hq, hk, dim
        counts = [cdiv(max(n, 0), page_rows) for n in lens]
        pages = sum(counts) + spare
        cols = max(max(counts), 1) if cols is None else cols
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int()
        self.where = list(range(b)) if slots is None else list(slots)
        n_slots = b if slots is None else max(max(slots) + 2, 1)
        table, all_lens, at = torch.full((n_slots, cols), -1, dtype=torch.int32), torch.zeros(n_slots, dtype=torch.int32), 0
        for i, w in enumerate(self.where):
            if w < 0 or w >= n_slots:
                continue
            table[w, :counts[i]] = order[at:at + counts[i]]
            all_lens[w] = lens[i]
            at += counts[i]
        self.table, self.lens = table.cuda(), all_lens.cuda()
        self.slot_of = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
        self.new_lens = None if news is None else torch.tensor(news, dtype=torch.int32, device="cuda")
        bad = float("nan") if poison else 0.0
        if layout == "rows":
            self.pools = [torch.full((pages, page_rows, hk, dim), bad, dtype=t, device="cuda") for _ in range(2)]
            self.k, self.v = self.pools
        elif layout == "heads":
            self.pools = [torch.full((pages, hk, page_rows, dim), bad, dtype=t, device="cuda") for _ in range(2)]
            self.k, self.v = (p.transpose(1, 2) for p in self.pools)
        elif layout == "joint":
            pool = torch.full((pages, 2, page_rows, hk, dim), bad, dtype=t, device="cuda")
            self.pools, self.k, self.v = [pool], pool[:, 0], pool[:, 1]
        else:
            assert layout == "padded"
            pools = [torch.full((pages, page_rows + 1, hk + 1, dim + 8), bad, dtype=t, device="cuda") for _ in range(2)]
            self.pools = pools
            self.k, self.v = pools[0][:, :page_rows, :hk, :dim], pools[1][:, 1:, 1:, 8:]
        if poison:
            self.v[:, ::2] = float("inf")
        self.q = (normal(b, rows, hq, dim) * spread).to(t)
        self.keys, self.values = [], []
        for i, w in enumerate(self.where):
            n = max(lens[i], 0)
            k, v = normal(n, hk, dim).to(t), normal(n, hk, dim).to(t)
            self.keys.append(k)
            self.values.append(v)
            if 0 <= w < n_slots and n:
                self.put(i, 0, k, v)

    def at(self, i, first, n):
        pos = torch.arange(first, first + n, device="cuda")
        return self.table[self.where[i]].long()[pos // self.page_rows], pos % self.page_rows

    def put(self, i, first, k, v):
        page, row = self.at(i, first, len(k))
        self.k[page, row] = k
        self.v[page, row] = v

    def shape(self, out, scale=None, k_new=None, v_new=None):
        return B.PagedShape.of(self.q, self.k, self.v, out, self.table, k_new, v_new, scale)

    def there(self):
        """Items that are there, with their number of new tokens."""
        return [(i, min(max(n, 0), self.rows)) for i, (w, n) in enumerate(zip(self.where, self.news_host))
                if 0 <= w < len(self.lens)]


def run(c, out, lse=None, scale=None, stream=None, scratch=None):
    shape = c.shape(out, scale)
    n = B.paged_attn_scratch_bytes(shape)
    if scratch is None:
        scratch = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    B.paged_attn(shape, c.q, c.k, c.v, c.table, c.lens, c.slot_of, c.new_lens, out, lse, scratch, n,
                 stream or torch.cuda.current_stream())
    if stream is None:
        code, detail = B.device_status(torch.cuda.current_stream())
        assert code == B.OK, hex(detail)
    assert bool((scratch[n:] == 0xFF).all())


def exact(c, i, n, scale, absent=()):
    """(O, lse, T = sum p |v|, A = scale sum |q||k|, sum |v|) of item i's n new tokens in 64 bits; `absent`: positions left out."""
    length, g = max(c.lens_host[i], 0), c.hq // c.hk
    q = c.q[i, :n].double().view(n, c.hk, g, c.dim).permute(1, 2, 0, 3)             # hk, g, n, dim
    k, v = (x.double().transpose(0, 1)[:, None] for x in (c.keys[i], c.values[i]))     # hk, 1, length, dim
    hidden = torch.arange(length, device="cuda") > length - n + torch.arange(n, device="cuda")[:, None]
    hidden[:, list(absent)] = True
    z = (scale * (q @ k.transpose(2, 3))).masked_fill(hidden, float("-inf"))
    lse = torch.logsumexp(z, 3) if length else torch.full((c.hk, g, n), float("-inf"), dtype=torch.float64, device="cuda")
    p = torch.exp(z - lse[..., None]).masked_fill(hidden, 0.0).nan_to_num(0.0)
    a = (scale * (q.abs() @ k.abs().transpose(2, 3))).masked_fill(hidden, 0.0).amax(3, keepdim=True) if length else \
        torch.zeros(c.hk, g, n, 1, dtype=torch.float64, device="cuda")
    sv = (~hidden).double() @ v.abs()
    back = lambda x: x.permute(2, 0, 1, 3).reshape(n, c.hq, -1)
    return back(p @ v), back(lse[..., None])[..., 0], back(p @ v.abs()), back(a), back(sv.expand(-1, g, -1, -1))


def check(c, lse=True, scale=None, absent=None):
    """One call against ``exact``.  Tolerances (u = 2^-24; h = half a step of the operands' type).  A score is a sum of dim
    products in fp32: off by (dim + 4) u A, which is a relative error of its exponential; exp2 adds 2^-21, and a part's weight
    exp(lse - max) 8 u (|lse| + 4) for the rounding of lse, twice over.  That enters numerator and denominator.  Probabilities
    are rounded once (h each; fp16 also loses 2^-25 of the row's maximum), products with V are added 16 at a time with up to 2 u each,
    the result is rounded once: |O - exact| <= h |O| + T (h + 2 rho + (n / 8 + 32) 2 u)."""
    b, t = len(c.where), TYPES[c.dtype]
    out = torch.full((b, c.rows, c.hq, c.dim), 7.0, dtype=t, device="cuda")
    got_lse = torch.full((b, c.hq, c.rows), 3.0, device="cuda") if lse else None
    run(c, out, got_lse, scale)
    sc = float(torch.tensor(c.dim ** -0.5 if scale is None else scale, dtype=torch.float32))
    h = torch.finfo(t).eps / 2
    left = torch.ones(b, c.rows, dtype=torch.bool, device="cuda")
    for i, n in c.there():
        left[i, :n] = False
        if n == 0:
            continue
        o, l64, tt, a, sv = exact(c, i, n, sc, () if absent is None else absent[i])
        length = max(c.lens_host[i], 0)
        have = torch.isfinite(l64)
        rho = (c.dim + 4) * U * a + 2.0 ** -21 + 8 * U * (l64.nan_to_num(0, 0, 0).abs()[..., None] + 4)
        tol = h * o.abs() * (1 + 2 * h) + tt * (h + 2 * rho + (length / 8 + 32) * 2 * U) * 1.01
        if c.dtype == "fp16":
            tol = tol + 2.0 ** -25 * sv + 2.0 ** -25
        err = (out[i, :n].double() - o).abs()
        assert bool((err <= tol + 1e-30).all()), (i, float((err / (tol + 1e-30)).max()))
        if lse:
            got = got_lse[i, :, :n].T
            assert torch.equal(got == float("-inf"), ~have), i
            ltol = rho[..., 0] + (length / 128 + 48) * U + 4 * U * l64.abs()
            assert bool(((got.double() - l64).abs() <= ltol)[have].all()), i
    assert bool((out[left] == 7.0).all())
    if lse:
        assert bool((got_lse.transpose(1, 2)[left] == 3.0).all())
    return out, got_lse
