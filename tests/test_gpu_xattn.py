"""Cross attention against the definition in 64 bits.

Tolerances (u = 2^-24; h = half a step of the operands' type, 2^-8 for bf16, 2^-11 for fp16).  A score
is a sum of head_dim products in fp32: off by (head_dim + 4) u A with A = scale sum |q||k|, which is a
relative error of its exponential; exp2 itself adds 2^-21.  That enters numerator and denominator.  The
probabilities are rounded once (h each; fp16 also loses 2^-25 of the row's maximum below its normal
range), the products with V are added 16 at a time with up to 2 u each, the result is rounded once.
T = sum_j p_j |v_j| carries all of it: |O - exact| <= h |O| + T (h + 2 rho + (n / 8 + 32) 2 u)."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def layout(kind, batch, rows, heads, dim, dtype, fill=float("nan")):
    """An empty (batch, rows, heads, dim) view of some layout inside a buffer of `fill`."""
    if kind == "rows":
        buf = torch.full((batch, rows, heads, dim), fill, dtype=dtype, device="cuda")
        return buf, buf
    if kind == "heads":
        buf = torch.full((batch, heads, rows, dim), fill, dtype=dtype, device="cuda")
        return buf, buf.transpose(1, 2)
    if kind == "rows first":
        buf = torch.full((rows, batch, heads, dim), fill, dtype=dtype, device="cuda")
        return buf, buf.transpose(0, 1)
    assert kind == "padded"
    buf = torch.full((batch, rows + 1, heads + 2, dim + 8), fill, dtype=dtype, device="cuda")
    return buf, buf[:, :rows, 1:heads + 1, :dim]


def operands(batch, q_rows, kv_rows, hq, hk, dim, dtype, lens=None, kind="rows", seed=0, spread=1.5, poison=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype]

    def make(rows, heads, s):
        buf, view = layout(kind, batch, rows, heads, dim, t)
        view.copy_((torch.randn(batch, rows, heads, dim, generator=g, device="cuda") * s).to(t))
        return view
    q, k, v = make(q_rows, hq, spread), make(kv_rows, hk, 1.0), make(kv_rows, hk, 1.0)
    lens_t = None
    if lens is not None:
        lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
        if poison:                            # what lies behind an item's states must not matter
            for b, n in enumerate(lens):
                n = min(max(n, 0), kv_rows)
                k[b, n:] = float("nan")
                v[b, n:] = float("inf")
                v[b, n + 1::2] = float("nan")
    return q, k, v, lens_t


def exact(q, k, v, lens, scale):
    """(O, lse, T, A, sum |v|) in 64 bits, item by item and head by head."""
    batch, q_rows, hq, dim = q.shape
    hk = k.shape[2]
    o = torch.zeros(batch, q_rows, hq, dim, dtype=torch.float64, device="cuda")
    t, sv = torch.zeros_like(o), torch.zeros_like(o)
    lse = torch.full((batch, hq, q_rows), float("-inf"), dtype=torch.float64, device="cuda")
    a = torch.zeros(batch, q_rows, hq, 1, dtype=torch.float64, device="cuda")
    for b in range(batch):
        n = k.shape[1] if lens is None else min(max(lens[b], 0), k.shape[1])
        if n == 0:
            continue
        for h in range(hq):
            kh = h // (hq // hk)
            qq, kk, vv = q[b, :, h].double(), k[b, :n, kh].double(), v[b, :n, kh].double()
            z = scale * (qq @ kk.T)
            lse[b, h] = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[b, h][:, None])
            o[b, :, h], t[b, :, h] = p @ vv, p @ vv.abs()
            sv[b, :, h] = vv.abs().sum(0)
            a[b, :, h, 0] = (scale * (qq.abs() @ kk.abs().T)).amax(1)
    return o, lse, t, a, sv


def run_forward(q, k, v, lens_t, out, want_lse=True, scale=None, stream=None):
    shape = B.XattnShape.of(q, k, v, out, scale)
    n = B.xattn_fwd_scratch_bytes(shape)
    scratch = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda") if n else None
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), 3.0, device="cuda") if want_lse else None
    B.xattn_fwd(shape, q, k, v, lens_t, out, lse, scratch, n, stream or torch.cuda.current_stream())
    code, detail = B.device_status(torch.cuda.current_stream())
    assert code == B.OK, hex(detail)
    if n:
        assert bool((scratch[n:] == 0xFF).all())
    return lse


def check_forward(batch, q_rows, kv_rows, hq, hk, dim, dtype, lens=None, kind="rows", scale=None, spread=1.5, want_lse=True,
                  seed=0):
    q, k, v, lens_t = operands(batch, q_rows, kv_rows, hq, hk, dim, dtype, lens, kind, seed, spread)
    buf, out = layout(kind, batch, q_rows, hq, dim, TYPES[dtype], 7.0)
    lse = run_forward(q, k, v, lens_t, out, want_lse, scale)
    sc = dim ** -0.5 if scale is None else scale
    sc = float(torch.tensor(sc, dtype=torch.float32))
    o, l64, t, a, sv = exact(q, k, v, lens, sc)
    h = torch.finfo(TYPES[dtype]).eps / 2
    rho = (dim + 4) * U * a + 2.0 ** -21
    tol = h * o.abs() * (1 + 2 * h) + t * (h + 2 * rho + (kv_rows / 8 + 32) * 2 * U) * (1 + 1e-2)
    if dtype == "fp16":
        tol = tol + 2.0 ** -25 * sv + 2.0 ** -25
    err = (out.double() - o).abs()
    assert bool((err <= tol + 1e-30).all()), float((err / (tol + 1e-30)).max())
    if want_lse:
        have = torch.isfinite(l64)
        assert torch.equal(lse == float("-inf"), ~have)
        rows_rho = rho.squeeze(3).transpose(1, 2)
        ltol = rows_rho + (kv_rows / 128 + 48) * U + 4 * U * l64.abs()
        assert bool(((lse.double() - l64).abs() <= ltol)[have].all())
    view = buf.clone()
    if kind == "padded":                       # the surroundings of the output
        view[:, :q_rows, 1:hq + 1, :dim] = 7.0
        assert bool((view == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 8, 32, 40, 72, 80])
def test_forward_one_block(dtype, dim):
    check_forward(1, 128, 128, 1, 1, dim, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("q_rows,kv_rows", [(17, 1), (128, 129), (129, 127), (256, 256), (257, 1000), (500, 333), (300, 2500),
                                            (20, 5000)])
@pytest.mark.parametrize("dim", [64, 128])
def test_forward_sizes(q_rows, kv_rows, dim, dtype):
    check_forward(2, q_rows, kv_rows, 2, 2, dim, dtype)


@pytest.mark.parametrize("kind", ["rows", "heads", "rows first", "padded"])
@pytest.mark.parametrize("q_rows", [1, 150])
def test_forward_layouts_shared_heads_and_lengths(kind, q_rows):
    check_forward(6, q_rows, 300, 8, 2, 64, "bf16", lens=[0, 1, 128, 129, 300, 299], kind=kind)
    check_forward(3, q_rows, 300, 4, 1, 96, "fp16", lens=[-5, 1000, 257], kind=kind)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [8, 32, 64, 80, 128])
@pytest.mark.parametrize("q_rows,hq,hk,kv_rows", [(1, 1, 1, 1), (1, 4, 4, 15), (1, 8, 1, 16), (1, 16, 1, 17), (3, 5, 1, 63),
                                                  (16, 2, 2, 65), (2, 8, 2, 4099), (1, 3, 3, 20000)])
def test_token_sizes(q_rows, hq, hk, kv_rows, dim, dtype):
    check_forward(2, q_rows, kv_rows, hq, hk, dim, dtype, want_lse=q_rows != 3)


def test_token_lengths():
    for hk in (1, 4):
        check_forward(9, 1, 1025, 4, hk, 64, "bf16", lens=[0, 1, 15, 16, 17, 64, 65, 1024, 1025])
        check_forward(9, 2, 700, 4, hk, 128, "fp16", lens=[0, 1, 15, 256, 17, 511, 65, 699, 700])


def test_no_states_at_all():
    for q_rows in (1, 40, 300):
        q = torch.randn(2, q_rows, 3, 64, device="cuda").bfloat16()
        k = torch.empty(2, 0, 3, 64, device="cuda", dtype=torch.bfloat16)
        out = torch.full_like(q, 9.0)
        lse = run_forward(q, k, k, None, out)
        assert bool((out == 0).all()) and bool((lse == float("-inf")).all())
        check_forward(3, q_rows, 200, 2, 2, 64, "bf16", lens=[0, 0, 0])


@pytest.mark.parametrize("q_rows", [1, 100])
def test_peaked_rows_growing_maxima_and_scales(q_rows):
    check_forward(1, q_rows, 1000, 2, 2, 64, "bf16", spread=12.0)
    check_forward(1, q_rows, 1000, 2, 2, 64, "fp16", spread=12.0, scale=0.5)
    check_forward(1, q_rows, 700, 2, 2, 128, "bf16", scale=0.0)
    # every block's maximum far above the last one's: the running maximum moves each time
    q = torch.ones(1, q_rows, 1, 64, device="cuda").bfloat16()
    k = (torch.arange(1000, device="cuda") / 8).floor()[None, :, None, None].expand(1, 1000, 1, 64).bfloat16().contiguous()
    v = torch.randn(1, 1000, 1, 64, device="cuda").bfloat16()
    out = torch.empty_like(q)
    run_forward(q, k, v, None, out)
    o, _, t, _, _ = exact(q, k, v, None, 0.125)
    assert bool(((out.double() - o).abs() <= 2.0 ** -8 * o.abs() + t * (2.0 ** -8 * 1.02 + 2e-3)).all())


@pytest.mark.parametrize("q_rows", [2, 130])
def test_values_that_are_not_finite_stay_in_their_rows(q_rows):
    q, k, v, _ = operands(2, q_rows, 300, 2, 2, 64, "bf16")
    clean = torch.empty_like(q)
    run_forward(q, k, v, None, clean)
    q[0, 1, 0] = float("nan")
    v[1, 7, 1, 3] = float("inf")
    out = torch.empty_like(q)
    run_forward(q, k, v, None, out)
    assert bool(out[0, 1, 0].isnan().all())
    assert not bool(out[1, :, 1, 3].isfinite().any())
    same = torch.ones_like(out, dtype=torch.bool)
    same[0, 1, 0] = False
    same[1, :, 1, 3] = False
    assert torch.equal(out[same], clean[same])


def test_more_than_32_bits_of_offset():
    """Rows 2^23 elements apart: the last key lies 2.5e9 elements into its buffer."""
    rows, stride = 300, 1 << 23
    buf = torch.empty(rows * stride + 64, dtype=torch.bfloat16, device="cuda")
    for q_rows in (1, 40):
        q = torch.randn(1, q_rows, 1, 64, device="cuda").bfloat16()
        k = torch.as_strided(buf, (1, rows, 1, 64), (rows * stride, stride, 64, 1))
        k.copy_(torch.randn(1, rows, 1, 64, device="cuda"))
        v = torch.as_strided(buf, (1, rows, 1, 64), (rows * stride, stride, 64, 1), 4096)[:, :rows]
        v.copy_(torch.randn(1, rows, 1, 64, device="cuda"))
        out, ref = torch.empty_like(q), torch.empty_like(q)
        run_forward(q, k, v, None, out)
        run_forward(q, k.contiguous(), v.contiguous(), None, ref)
        assert torch.equal(out, ref)


def test_replay_streams_and_repeatability():
    cases = [operands(2, r, 3000, 4, 2, 64, "bf16", [3000, 1777], poison=False, seed=r) for r in (1, 200)]
    for q, k, v, lens in cases:
        first = torch.empty_like(q)
        run_forward(q, k, v, lens, first)
        shape = B.XattnShape.of(q, k, v, first)
        n = B.xattn_fwd_scratch_bytes(shape)
        assert n > 0                              # both are split over the keys
        out, side_out = torch.empty_like(q), torch.empty_like(q)
        s1, s2 = (torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2))
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph):
            B.xattn_fwd(shape, q, k, v, lens, out, None, s1, n, torch.cuda.current_stream())
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            graph.replay()
            B.xattn_fwd(shape, q, k, v, lens, side_out, None, s2, n, side)
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(side_out, first)


def test_waits_that_run_out_end_the_kernel():
    """Nothing is loaded, so every wait runs out after a millisecond: the kernel returns, the status
    says so, and the next call is right."""
    q, k, v, _ = operands(1, 300, 500, 2, 2, 64, "bf16")
    out, ref = torch.empty_like(q), torch.empty_like(q)
    run_forward(q, k, v, None, ref)
    shape = B.XattnShape.of(q, k, v, out)
    n = B.xattn_fwd_scratch_bytes(shape)
    scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    try:
        B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 1_000_000)
        B.debug_set(B.DEBUG_SKIP_NEXT_XATTN_LOADS, 1)
        B.xattn_fwd(shape, q, k, v, None, out, None, scratch, n, torch.cuda.current_stream())
        assert B.device_status(torch.cuda.current_stream())[0] == B.ERR_DEVICE_TIMEOUT
    finally:
        B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 0)
        B.debug_set(B.DEBUG_SKIP_NEXT_XATTN_LOADS, 0)
    run_forward(q, k, v, None, out)
    assert torch.equal(out, ref)


# ------------------------------------------------------------------ backward --
def exact_backward(q, k, v, lens, o, lse, do, scale, dtype):
    """(value, tolerance) of dQ, dK, dV in 64 bits from the operands as they are.  An entry of dS is off by
    P (W (dim + 4) u + |dP - delta| (rho + 2 u)), W = sum |dO||V| + sum |dO||O|, and by its rounding; then the
    products' sums as in the forward direction."""
    h = torch.finfo(TYPES[dtype]).eps / 2
    small = 2.0 ** -25 if dtype == "fp16" else 0.0
    batch, q_rows, hq, dim = q.shape
    kv_rows, hk = k.shape[1], k.shape[2]
    zeros = lambda t: torch.zeros(t.shape, dtype=torch.float64, device="cuda")
    (dq, dk, dv), (tq, tk, tv) = (zeros(q), zeros(k), zeros(v)), (zeros(q), zeros(k), zeros(v))
    for b in range(batch):
        n = kv_rows if lens is None else min(max(lens[b], 0), kv_rows)
        if n == 0:
            continue
        for hh in range(hq):
            kh = hh // (hq // hk)
            qq, kk, vv = q[b, :, hh].double(), k[b, :n, kh].double(), v[b, :n, kh].double()
            oo, dd, ll = o[b, :, hh].double(), do[b, :, hh].double(), lse[b, hh].double()[:, None]
            z = scale * (qq @ kk.T)
            p = torch.exp(z - ll)
            delta = (dd * oo).sum(1, keepdim=True)
            diff = dd @ vv.T - delta
            ds = p * diff
            dq[b, :, hh] = scale * (ds @ kk)
            dk[b, :n, kh] += scale * (ds.T @ qq)
            dv[b, :n, kh] += p.T @ dd
            w = dd.abs() @ vv.abs().T + (dd.abs() * oo.abs()).sum(1, keepdim=True)
            rho = (dim + 4) * U * scale * (qq.abs() @ kk.abs().T) + 4 * U * (z.abs() + ll.abs()) + 2.0 ** -21
            e = p * (w * (dim + 4) * U + diff.abs() * (rho + 2 * U))
            e = e + h * (ds.abs() + e) + small
            rows = (max(n, q_rows * (hq // hk)) / 8 + 32) * 2 * U
            tq[b, :, hh] = scale * ((e + rows * ds.abs()) @ kk.abs())
            tk[b, :n, kh] += scale * ((e + rows * ds.abs()).T @ qq.abs())
            tv[b, :n, kh] += (p * (rho + h * (1 + rho) + rows) + small).T @ dd.abs()
    return [(g, (t + h * (g.abs() + t)) * 1.01 + 1e-30 + small) for g, t in ((dq, tq), (dk, tk), (dv, tv))]


def check_backward(batch, q_rows, kv_rows, hq, hk, dim, dtype, lens=None, kind="rows", scale=None, spread=1.5, keys_too=True,
                   seed=0):
    t = TYPES[dtype]
    q, k, v, lens_t = operands(batch, q_rows, kv_rows, hq, hk, dim, dtype, lens, kind, seed, spread)
    sc = float(torch.tensor(dim ** -0.5 if scale is None else scale, dtype=torch.float32))
    o64, lse64, _, _, _ = exact(q, k, v, lens, sc)
    _, o = layout(kind, batch, q_rows, hq, dim, t)
    _, do = layout(kind, batch, q_rows, hq, dim, t)
    o.copy_(o64.to(t))
    do.copy_((torch.randn(batch, q_rows, hq, dim, generator=torch.Generator(device="cuda").manual_seed(seed + 1),
                          device="cuda")).to(t))
    lse = lse64.float()
    bufs = [layout(kind, batch, r, hh, dim, t, 7.0) for r, hh in ((q_rows, hq), (kv_rows, hk), (kv_rows, hk))]
    shape = B.XattnShape.of(q, k, v, o, scale)
    n = B.xattn_bwd_scratch_bytes(shape)
    scratch = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    grads = [g for _, g in bufs]
    B.xattn_bwd(shape, q, k, v, lens_t, o, lse, do, grads[0], *(grads[1:] if keys_too else (None, None)), scratch, n,
                torch.cuda.current_stream())
    code, detail = B.device_status(torch.cuda.current_stream())
    assert code == B.OK, hex(detail)
    assert bool((scratch[n:] == 0xFF).all())
    if not keys_too:
        assert all(bool((b == 7.0).all()) for b, _ in bufs[1:])
    ref = exact_backward(q, k, v, lens, o, lse, do, sc, dtype)
    for name, got, (want, tol) in list(zip(("dq", "dk", "dv"), grads, ref))[:3 if keys_too else 1]:
        err = (got.double() - want).abs()
        assert bool((err <= tol).all()), (name, float((err / tol).nan_to_num(nan=1e9).max()))
    if lens is not None and keys_too:
        for b, m in enumerate(lens):
            m = min(max(m, 0), kv_rows)
            assert bool((grads[1][b, m:] == 0).all()) and bool((grads[2][b, m:] == 0).all())
    if kind == "padded":
        for (buf, _), (r, hh) in zip(bufs, ((q_rows, hq), (kv_rows, hk), (kv_rows, hk))):
            around = buf.clone()
            around[:, :r, 1:hh + 1, :dim] = 7.0
            assert bool((around == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 8, 32, 40, 72, 80])
def test_backward_one_block(dtype, dim):
    check_backward(1, 128, 128, 1, 1, dim, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("q_rows,kv_rows", [(1, 1), (1, 700), (700, 1), (128, 129), (129, 127), (256, 256), (257, 1000),
                                            (500, 333), (2000, 400)])
@pytest.mark.parametrize("dim", [64, 128])
def test_backward_sizes(q_rows, kv_rows, dim, dtype):
    check_backward(2, q_rows, kv_rows, 2, 2, dim, dtype)


@pytest.mark.parametrize("kind", ["rows", "heads", "rows first", "padded"])
def test_backward_layouts_shared_heads_and_lengths(kind):
    check_backward(6, 150, 300, 8, 2, 64, "bf16", lens=[0, 1, 128, 129, 300, 299], kind=kind)
    check_backward(3, 150, 300, 4, 1, 96, "fp16", lens=[-5, 1000, 257], kind=kind)


def test_backward_many_blocks_and_optional_gradients():
    check_backward(1, 1500, 3000, 1, 1, 128, "bf16")
    check_backward(1, 1500, 1000, 6, 2, 64, "fp16", lens=[901])
    check_backward(2, 300, 300, 2, 2, 64, "bf16", keys_too=False)
    check_backward(1, 200, 300, 2, 2, 64, "bf16", scale=0.0)
    check_backward(1, 200, 300, 2, 2, 64, "bf16", spread=10.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_backward_split_over_the_long_axis(dtype):
    """Few queries against many states and the other way round: parts that are added afterwards, some of them
    without states or queries of their own."""
    check_backward(1, 20, 3000, 2, 1, 64, dtype)
    check_backward(1, 2500, 30, 2, 1, 64, dtype)
    check_backward(3, 70, 2000, 2, 2, 128, dtype, lens=[2000, 1, 700], kind="padded")
    check_backward(2, 1800, 130, 4, 2, 80, dtype, lens=[130, 0], kind="heads")
    check_backward(1, 40, 1500, 1, 1, 32, dtype, keys_too=False)


def test_backward_without_queries_or_states():
    empty = torch.empty(2, 0, 3, 64, device="cuda", dtype=torch.bfloat16)
    some = torch.randn(2, 200, 3, 64, device="cuda").bfloat16()
    lse = torch.full((2, 3, 200), float("-inf"), device="cuda")
    scratch = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream()
    dk, dv = torch.full_like(some, 5.0), torch.full_like(some, 5.0)
    B.xattn_bwd(B.XattnShape.of(empty, some, some, empty), None, some, some, None, None, None, None, None, dk, dv, None, 0, stream)
    assert bool((dk == 0).all()) and bool((dv == 0).all())
    dq = torch.full_like(some, 5.0)
    B.xattn_bwd(B.XattnShape.of(some, empty, empty, some), some, None, None, None, some, lse, some, dq, None, None, scratch,
                1 << 16, stream)
    assert bool((dq == 0).all())


def test_backward_formula_against_differences():
    """The 64-bit gradients that the kernels are compared with, against central differences of the forward
    definition (step 1e-6: differences are exact to about 1e-8) with unrounded O and lse."""
    q, k, v, _ = operands(1, 5, 7, 2, 1, 8, "bf16")
    q, k, v = q.double(), k.double(), v.double()
    sc, w = 0.35, torch.randn(1, 5, 2, 8, device="cuda", dtype=torch.float64)
    o, lse, _, _, _ = exact(q, k, v, [6], sc)
    ref = exact_backward(q, k, v, [6], o, lse, w, sc, "bf16")
    for i, x in enumerate((q, k, v)):
        for at in ((0, 0, 0, 0), (0, 3, x.shape[2] - 1, 5), (0, x.shape[1] - 1, 0, 7)):
            up, down = [t.clone() for t in (q, k, v)], [t.clone() for t in (q, k, v)]
            up[i][at] += 1e-6
            down[i][at] -= 1e-6
            slope = float(((exact(*up, [6], sc)[0] - exact(*down, [6], sc)[0]) * w).sum() / 2e-6)
            assert abs(slope - float(ref[i][0][at])) < 1e-6


def test_backward_replay_streams_and_repeatability():
    q, k, v, lens = operands(2, 300, 500, 4, 2, 64, "bf16", [500, 377], poison=False)
    o = torch.empty_like(q)
    lse = run_forward(q, k, v, lens, o)
    do = torch.randn_like(q)
    shape = B.XattnShape.of(q, k, v, o)
    n = B.xattn_bwd_scratch_bytes(shape)

    def grads():
        return [torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty(n, dtype=torch.uint8, device="cuda")]

    def call(g, stream):
        B.xattn_bwd(shape, q, k, v, lens, o, lse, do, g[0], g[1], g[2], g[3], n, stream)

    first, replayed, other = grads(), grads(), grads()
    call(first, torch.cuda.current_stream())
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        call(replayed, torch.cuda.current_stream())
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        call(other, side)
    torch.cuda.synchronize()
    for a, b, c in zip(first[:3], replayed, other):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_backward_waits_that_run_out_end_the_kernel():
    q, k, v, _ = operands(1, 300, 500, 2, 2, 64, "bf16")
    o = torch.empty_like(q)
    lse = run_forward(q, k, v, None, o)
    shape = B.XattnShape.of(q, k, v, o)
    n = B.xattn_bwd_scratch_bytes(shape)
    scratch = torch.empty(n, dtype=torch.uint8, device="cuda")
    out = [[torch.empty_like(t) for t in (q, k, v)] for _ in range(2)]
    stream = torch.cuda.current_stream()
    B.xattn_bwd(shape, q, k, v, None, o, lse, q, *out[0], scratch, n, stream)
    try:
        B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 1_000_000)
        B.debug_set(B.DEBUG_SKIP_NEXT_XATTN_LOADS, 1)
        B.xattn_bwd(shape, q, k, v, None, o, lse, q, *out[1], scratch, n, stream)
        assert B.device_status(stream)[0] == B.ERR_DEVICE_TIMEOUT
    finally:
        B.debug_set(B.DEBUG_WAIT_LIMIT_NS, 0)
        B.debug_set(B.DEBUG_SKIP_NEXT_XATTN_LOADS, 0)
    B.xattn_bwd(shape, q, k, v, None, o, lse, q, *out[1], scratch, n, stream)
    assert B.device_status(stream)[0] == B.OK
    assert all(torch.equal(a, b) for a, b in zip(*out))
