"""LayerNorm over rows, forward and backward, against the definition in 64 bits.

Tolerances (u = 2^-24, one fp32 rounding).  A row's sums are added by at most kDepth(n) terms in a
row (a thread's own elements, then the joins), so each of them is off by at most kDepth u times the
sum of its terms' magnitudes.  Forward: the mean's error in units of the spread is kDepth u
(E|x - mean| <= spread), the variance's relative error (kDepth + 4) u, the output adds a handful of
roundings of |z|, |gamma| and |beta|; then one rounding to the row's type.  Backward likewise."""
import pytest
import torch

from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {B.F32: torch.float32, B.BF16: torch.bfloat16, B.F16: torch.float16}


def depth(n):
    """Terms added one after the other: per-thread elements (32 in registers, n / 1024 beyond) and joins."""
    return max(32, n // 1024 + 1) + 12


def half_step(dtype, ref):
    t = TYPES[dtype]
    return torch.finfo(t).eps / 2 * ref.abs() + (2.0 ** -25 if t == torch.float16 else 1e-38)


def matrix(rows, n, ld, dtype, seed, lead=0, mean=0.0, spread=1.0, fill=None):
    """rows x n view of pitch ld, `lead` elements into a buffer filled with `fill` (default NaN)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((lead + max(rows * ld, 1) + 8,), float("nan") if fill is None else fill, dtype=TYPES[dtype], device="cuda")
    view = torch.as_strided(buf, (rows, n), (ld, 1), lead)
    if fill is None:
        rowmean = mean + torch.randn(rows, 1, generator=g, device="cuda") * spread
        view.copy_((torch.randn(rows, n, generator=g, device="cuda") * spread + rowmean).to(TYPES[dtype]))
    return buf, view


def vector(n, dtype, seed, around=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (around + 0.3 * torch.randn(n, generator=g, device="cuda")).to(TYPES[dtype])


def forward64(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    z = (x - mean) * rstd
    y = z if gamma is None else z * gamma.double()
    return (y if beta is None else y + beta.double()), mean[:, 0], rstd[:, 0], z


def check_forward(rows, n, dtype, pdtype, ldx=None, ldy=None, lead=0, with_params=True, in_place=False, stats=True,
                  eps=1e-5, mean=0.0, spread=1.0):
    ldx, ldy = ldx or n, ldy or n
    xbuf, x = matrix(rows, n, ldx, dtype, 1, lead, mean, spread)
    gamma = vector(n, pdtype, 2, 1.0) if with_params else None
    beta = vector(n, pdtype, 3) if with_params else None
    ref, rmean, rrstd, z = forward64(x, gamma, beta, eps)
    ybuf, y = (xbuf, x) if in_place else matrix(rows, n, ldy, dtype, 0, lead, fill=7.0)
    m = torch.full((rows,), -1.0, device="cuda") if stats else None
    r = torch.full((rows,), -1.0, device="cuda") if stats else None
    before = ybuf.clone()
    B.layernorm_rows(x.data_ptr(), gamma, beta, y.data_ptr(), m, r, rows, n, ldx, ldx if in_place else ldy, dtype,
                     pdtype, eps, torch.cuda.current_stream())
    c = depth(n)
    ga = 1.0 if gamma is None else gamma.double().abs()
    be = 0.0 if beta is None else beta.double().abs()
    tol = half_step(dtype, ref) * (1 + 1e-3) + U * (c * (z.abs() + 1) * ga + 8 * (z.abs() * ga + be))
    err = (y.double() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    if stats:
        sd = (x.double() if not in_place else before.as_strided((rows, n), (ldx, 1), lead).double()).std(1, unbiased=False)
        assert bool(((m.double() - rmean).abs() <= U * (2 * rmean.abs() + c * sd) + 1e-38).all())
        assert bool(((r.double() - rrstd).abs() <= U * (c + 8) * rrstd).all())
    # padding columns, and what lies before and behind the matrix, as they were
    after = ybuf.clone()
    after.as_strided((rows, n), (ldx if in_place else ldy, 1), lead).zero_()
    before.as_strided((rows, n), (ldx if in_place else ldy, 1), lead).zero_()
    assert torch.equal(after.view(torch.uint8), before.view(torch.uint8))


LENGTHS = [1, 2, 7, 8, 33, 255, 256, 264, 1000, 1024, 1025, 1537, 2048, 2056, 4096, 4104, 5001, 8192, 8200, 16384,
           16392, 20001]


@pytest.mark.parametrize("dtype", [B.F32, B.BF16, B.F16])
@pytest.mark.parametrize("n", LENGTHS)
def test_forward_lengths(n, dtype):
    check_forward(5, n, dtype, dtype if n % 2 else B.F32)


@pytest.mark.parametrize("dtype,n,rows", [(B.BF16, 64, 20011), (B.F32, 1024, 3001), (B.F16, 4096, 1500), (B.BF16, 1537, 700),
                                          (B.F32, 200, 1), (B.BF16, 16384, 301), (B.F32, 17000, 400)])
def test_forward_many_rows(dtype, n, rows):
    check_forward(rows, n, dtype, B.F32)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_forward_pitches_offsets_and_optional_operands(dtype):
    check_forward(7, 100, dtype, dtype, ldx=104, ldy=112)
    check_forward(7, 96, dtype, dtype, ldx=104, ldy=96, lead=8)
    check_forward(7, 96, dtype, dtype, ldx=97, ldy=101, lead=3)
    check_forward(7, 2000, dtype, B.F32, ldx=2048, ldy=2001)
    check_forward(7, 1024, dtype, dtype, with_params=False, stats=False)
    check_forward(9, 3000, dtype, dtype, in_place=True)
    check_forward(9, 99, dtype, dtype, ldx=101, in_place=True)
    check_forward(3, 17003, dtype, dtype, ldx=17010, in_place=True)


@pytest.mark.parametrize("n", [500, 5000, 20000])
def test_forward_mean_far_above_the_spread(n):
    # x - mean is exact to fp32's step at 4096 (2^-11 of the spread); the output must still be right for that x
    check_forward(5, n, B.F32, B.F32, mean=4096.0, spread=2.0 ** -3)
    check_forward(5, n, B.F32, B.F32, mean=-1e6, spread=1.0)


def test_forward_constant_rows_and_non_finite_rows():
    n = 300
    for width in (n, 20000):
        x = torch.full((6, width), 3.5, device="cuda")
        x[1, 7] = float("nan")
        x[2, 5] = float("inf")
        x[3] = torch.randn(width, device="cuda")
        y = torch.empty_like(x)
        B.layernorm_rows(x, None, None, y, None, None, 6, width, width, width, B.F32, B.F32, 1e-5, torch.cuda.current_stream())
        assert bool((y[[0, 4, 5]] == 0).all())
        assert bool(y[1].isnan().all()) and bool(y[2].isnan().all())
        assert bool(y[3].isfinite().all())


def backward64(dy, x, gamma, mean, rstd):
    n = x.shape[1]
    z = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy.double() * (1.0 if gamma is None else gamma.double())
    c1, c2 = g.sum(1, keepdim=True) / n, (g * z).sum(1, keepdim=True) / n
    dx = rstd.double()[:, None] * (g - c1 - z * c2)
    return dx, (dy.double() * z).sum(0), dy.double().sum(0), z, g


def check_backward(rows, n, dtype, pdtype, ld=(None, None, None), lead=0, with_gamma=True, want=(True, True, True),
                   over=None):
    lddy, ldx, lddx = (v or n for v in ld)
    xbuf, x = matrix(rows, n, ldx, dtype, 11, lead)
    dybuf, dy = matrix(rows, n, lddy, dtype, 12, lead, spread=0.1)
    gamma = vector(n, pdtype, 13, 1.0) if with_gamma else None
    _, m64, r64, _ = forward64(x, None, None, 1e-5)
    mean, rstd = m64.float(), r64.float()
    dx64, dg64, db64, z, g = backward64(dy, x, gamma, mean, rstd)
    dyc = dy.double()
    if over == "x":
        dxbuf, dx, lddx = xbuf, x, ldx
    elif over == "dy":
        dxbuf, dx, lddx = dybuf, dy, lddy
    else:
        dxbuf, dx = matrix(rows, n, lddx, dtype, 0, lead, fill=5.0)
    before = dxbuf.clone()
    dg = torch.full((n,), 9.0, dtype=TYPES[pdtype], device="cuda") if want[1] else None
    db = torch.full((n,), 9.0, dtype=TYPES[pdtype], device="cuda") if want[2] else None
    size = B.layernorm_rows_bwd_scratch_bytes(rows, n)
    scratch = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN patterns
    B.layernorm_rows_bwd(dy.data_ptr(), x.data_ptr(), gamma, mean, rstd, dx.data_ptr() if want[0] else None, dg, db,
                         rows, n, lddy, ldx, lddx, dtype, pdtype, scratch if dg is not None or db is not None else None,
                         size, torch.cuda.current_stream())
    assert bool((scratch[size:] == 0xFF).all())
    c = depth(n)
    if want[0]:
        mg, mgz = g.abs().mean(1, keepdim=True), (g * z).abs().mean(1, keepdim=True)
        tol = half_step(dtype, dx64) * (1 + 1e-3) + U * rstd.double()[:, None] * (
            c * (mg + z.abs() * mgz) + 8 * (g.abs() + mg + z.abs() * mgz) + 4 * z.abs() * mgz)
        err = (dx.double() - dx64).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
    # column sums: at most rows / 148 + 1 rows one after the other (fewer CTAs than 148 only when there are fewer
    # rows), then up to 1184 partial sums, 37 and 32 at a time
    cd = rows / 148 + 1 + 8 + 37 + 32 + 8
    for got, ref, mag in ((dg, dg64, (dyc * z).abs().sum(0)), (db, db64, dyc.abs().sum(0))):
        if got is not None:
            tol = half_step(pdtype, ref) * (1 + 1e-3) + U * (cd + 4) * mag + 1e-30
            err = (got.double() - ref).abs()
            assert bool((err <= tol).all()), float((err / tol).max())
    if want[0]:
        after = dxbuf.clone()
        after.as_strided((rows, n), (lddx, 1), lead).zero_()
        before.as_strided((rows, n), (lddx, 1), lead).zero_()
        assert torch.equal(after.view(torch.uint8), before.view(torch.uint8))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16, B.F16])
@pytest.mark.parametrize("n", LENGTHS)
def test_backward_lengths(n, dtype):
    check_backward(5, n, dtype, dtype if n % 2 else B.F32)


@pytest.mark.parametrize("dtype,n,rows", [(B.BF16, 64, 20011), (B.F32, 1024, 3001), (B.F16, 4096, 1500), (B.BF16, 1537, 700),
                                          (B.F32, 200, 1), (B.BF16, 16384, 301), (B.F32, 17000, 400), (B.BF16, 2048, 2000)])
def test_backward_many_rows(dtype, n, rows):
    check_backward(rows, n, dtype, B.F32)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_backward_pitches_offsets_and_optional_gradients(dtype):
    check_backward(7, 96, dtype, dtype, ld=(104, 112, 120))
    check_backward(7, 96, dtype, dtype, ld=(97, 99, 101), lead=3)
    check_backward(300, 1000, dtype, dtype, with_gamma=False)
    for want in ((True, False, False), (False, True, False), (False, False, True), (False, True, True)):
        check_backward(9, 200, dtype, dtype, want=want)
        check_backward(9, 17001, dtype, dtype, want=want)
    for n in (200, 3000, 17001):
        check_backward(9, n, dtype, dtype, over="x")
        check_backward(9, n, dtype, dtype, over="dy")


def test_backward_without_rows_gives_zero_weight_gradients():
    dg, db = torch.full((100,), 3.0, device="cuda"), torch.full((100,), 3.0, device="cuda")
    size = B.layernorm_rows_bwd_scratch_bytes(0, 100)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    B.layernorm_rows_bwd(None, None, None, None, None, None, dg, db, 0, 100, 100, 100, 100, B.F32, B.F32, scratch, size,
                         torch.cuda.current_stream())
    assert bool((dg == 0).all()) and bool((db == 0).all())


def test_gradient_against_differences():
    """dx and dgamma against central differences of the 64-bit forward definition (step 1e-5: the
    differences are exact to about 1e-9, the fp32 gradients to about 1e-6)."""
    rows, n, h = 3, 24, 1e-5
    _, x = matrix(rows, n, n, B.F32, 21)
    gamma, beta, w = vector(n, B.F32, 22, 1.0), vector(n, B.F32, 23), torch.randn(rows, n, device="cuda", dtype=torch.float64)
    _, m, r, _ = forward64(x, gamma, beta, 1e-5)
    loss = lambda xx, gg: float((forward64(xx, gg, beta, 1e-5)[0] * w).sum())
    dx, dg, db = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    size = B.layernorm_rows_bwd_scratch_bytes(rows, n)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    B.layernorm_rows_bwd(w.float(), x, gamma, m.float(), r.float(), dx, dg, db, rows, n, n, n, n, B.F32, B.F32, scratch, size,
                         torch.cuda.current_stream())
    for i, j in ((0, 0), (1, 7), (2, 23)):
        e = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
        e[i, j] = h
        assert abs((loss(x.double() + e, gamma) - loss(x.double() - e, gamma)) / (2 * h) - float(dx[i, j])) < 1e-4
        assert abs((loss(x, gamma.double() + e[i]) - loss(x, gamma.double() - e[i])) / (2 * h) - float(dg[j])) < 1e-4


@pytest.mark.parametrize("n", [24, 40, 64, 99, 128, 200, 256, 333, 512, 1000, 1001, 1024])
@pytest.mark.parametrize("dtype", [B.F32, B.BF16, B.F16])
def test_short_rows_by_the_thousand(n, dtype):
    """Rows enough for the kernels that give a row to a part of a warp, the last round of rows not full."""
    check_forward(4999, n, dtype, dtype, in_place=n == 200)
    check_backward(4999, n, dtype, dtype)


def test_graph_replay_side_stream_and_repeatability():
    rows, n = 700, 1537
    _, x = matrix(rows, n, n, B.BF16, 31)
    _, dy = matrix(rows, n, n, B.BF16, 32)
    gamma, beta = vector(n, B.F32, 33, 1.0), vector(n, B.F32, 34)
    size = B.layernorm_rows_bwd_scratch_bytes(rows, n)

    def buffers():
        return dict(y=torch.empty_like(x), mean=torch.empty(rows, device="cuda"), rstd=torch.empty(rows, device="cuda"),
                    dx=torch.empty_like(x), dg=torch.empty(n, device="cuda"), db=torch.empty(n, device="cuda"),
                    scratch=torch.empty(size, dtype=torch.uint8, device="cuda"))

    def step(b, stream):
        B.layernorm_rows(x, gamma, beta, b["y"], b["mean"], b["rstd"], rows, n, n, n, B.BF16, B.F32, 1e-5, stream)
        B.layernorm_rows_bwd(dy, x, gamma, b["mean"], b["rstd"], b["dx"], b["dg"], b["db"], rows, n, n, n, n, B.BF16, B.F32,
                             b["scratch"], size, stream)

    eager, replayed, other = buffers(), buffers(), buffers()
    step(eager, torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed, torch.cuda.current_stream())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):                    # a replay and an eager call of another stream at the same time
        graph.replay()
        step(other, side)
    torch.cuda.synchronize()
    for key in ("y", "mean", "rstd", "dx", "dg", "db"):
        assert torch.equal(eager[key], replayed[key]) and torch.equal(eager[key], other[key]), key
