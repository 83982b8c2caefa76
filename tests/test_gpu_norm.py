"""Layer norm of feature rows, forward and backward, against the formulas in 64 bits.

Tolerances.  u is half a unit in the last place of the rows' type (2^-11 fp16, 2^-8 bf16, 2^-24 fp32): the one rounding of an output.  Sums of
a row are trees of at most 32 + 8 fp32 additions, 2^-18 of the sum of magnitudes; a column sum is a chain of at most some 200 additions for
the sizes here, 2^-16 of the sum of magnitudes."""
import pytest
import torch

from paper_2511_20834_amd import binding as B

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
U = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}
TINY = {F16: 2.0 ** -24, BF16: 0.0, F32: 0.0}  # spacing of fp16 near zero
EPS = 1e-5


def rows(n, c, dtype, gen, pitch=0, first=0):
    """n x c values, as columns [first, first + c) of rows of `pitch` elements."""
    t = (torch.randn(n, c, generator=gen) * (0.5 + torch.rand(c, generator=gen)) + torch.randn(c, generator=gen)).to(dtype).cuda()
    if not pitch:
        return t
    wide = torch.full((n, pitch), float("nan"), dtype=dtype, device="cuda")
    wide[:, first:first + c] = t
    return wide[:, first:first + c]


def within(got, ref, tol, what):
    got, tol = got.double().cpu(), tol.cpu()
    over = (got - ref.cpu()).abs() - tol
    assert torch.isfinite(got).all() and over.max() <= 0, (what, float(over.max()), int(over.argmax()))


def forward_ref(x, r, gamma, beta, eps):
    z = x.double() if r is None else x.double() + r.double()
    mean, var = z.mean(1), z.var(1, correction=0)
    rstd = (var + eps) ** -0.5
    h = (z - mean[:, None]) * rstd[:, None]
    g = 1.0 if gamma is None else gamma.double()
    return z, mean, rstd, h, h * g + (0.0 if beta is None else beta.double())


SHAPES = [(1, 1), (3, 2), (1, 64), (257, 5), (33, 90), (700, 16), (129, 24), (65, 100), (1000, 64), (77, 257), (40, 512), (31, 513), (9, 1024), (5, 2048),
          (6, 2050), (3, 2051), (4, 4099), (2, 8192), (3, 8191)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("extra,pitch,first", [(False, 0, 0), (True, 8, 0), (True, 1, 1), (False, 6, 2)])
def test_forward(n, c, dtype, extra, pitch, first):
    gen = torch.Generator().manual_seed(n * 10007 + c)
    p = c + pitch if pitch else 0
    x, r = rows(n, c, dtype, gen, p, first), rows(n, c, dtype, gen, p, first) if extra else None
    gamma, beta = (1 + torch.randn(c, generator=gen)).cuda(), torch.randn(c, generator=gen).cuda()
    out = torch.full((n, c + pitch + 3), 7.0, dtype=dtype, device="cuda")
    y, s, mean, rstd = B.spc_layer_norm_forward(x, gamma, beta, eps=EPS, residual=r, want_stats=True, out=out[:, first:first + c])
    z, m, rs, h, ref = forward_ref(x, r, gamma, beta, EPS)
    mag = z.abs().mean(1)
    within(mean, m, 2.0 ** -18 * mag, "mean")
    # (the variance of a row is off by its own rounding and by the mean's, squared)
    within(rstd, rs, 2.0 ** -17 * rs * (1 + (2.0 ** -18 * mag * rs) ** 2 * 2.0 ** 17), "rstd")
    tol = U[dtype] * ref.abs() + TINY[dtype] + 2.0 ** -16 * (gamma.double().abs() * (h.abs() + (mag * rs)[:, None] + 1) + beta.double().abs())
    within(y, ref, tol, "y")
    if extra:
        within(s, z, U[dtype] * z.abs() + TINY[dtype] + 2.0 ** -23 * z.abs(), "sum")
    else:
        assert s is None
    assert (out[:, :first] == 7).all() and (out[:, first + c:] == 7).all()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("n,c", SHAPES + [(0, 64), (6011, 128), (20_000, 36)])
@pytest.mark.parametrize("extra,pitch,first", [(False, 0, 0), (True, 8, 0), (True, 1, 1), (False, 6, 2)])
def test_backward(n, c, dtype, extra, pitch, first):
    gen = torch.Generator().manual_seed(n * 10007 + c + 1)
    p = c + pitch if pitch else 0
    x, dy, e = rows(n, c, dtype, gen, p, first), rows(n, c, dtype, gen, p, first), rows(n, c, dtype, gen, p, first) if extra else None
    gamma = (1 + torch.randn(c, generator=gen)).cuda()
    _, mean, rstd, _, _ = forward_ref(x, None, None, None, EPS)
    mean, rstd = mean.float(), rstd.float()
    dx, dgamma, dbeta = B.spc_layer_norm_backward(dy, x, mean, rstd, gamma, dsum=e)
    s = rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * s
    dh = 2.0 ** -22 * (x.double().abs() + mean.double().abs()[:, None]) * s  # rounding of h
    w = dy.double() * gamma.double()
    ref = s * (w - w.mean(1, keepdim=True) - h * (w * h).mean(1, keepdim=True)) + (e.double() if extra else 0.0)
    wm, wh = w.abs().mean(1, keepdim=True), (w * h).abs().mean(1, keepdim=True)
    lost = 2.0 ** -16 * s * (w.abs() + wm + h.abs() * wh) + s * (dh * wh + h.abs() * (w.abs() * dh).mean(1, keepdim=True))
    within(dx, ref, U[dtype] * ref.abs() + TINY[dtype] + lost + 2.0 ** -23 * ref.abs(), "dx") if n else None
    within(dgamma, (dy.double() * h).sum(0), 2.0 ** -16 * (dy.double() * h).abs().sum(0) + (dy.double().abs() * dh).sum(0), "dgamma")
    within(dbeta, dy.double().sum(0), 2.0 ** -16 * dy.double().abs().sum(0), "dbeta")


def test_gradients_against_differences():
    """The fp32 backward pass along random directions against central differences of the forward pass in 64 bits."""
    gen = torch.Generator().manual_seed(3)
    n, c = 50, 33
    x, r, dy, e = (rows(n, c, F32, gen) for _ in range(4))
    gamma, beta = (1 + torch.randn(c, generator=gen)).cuda(), torch.randn(c, generator=gen).cuda()
    _, total, mean, rstd = B.spc_layer_norm_forward(x, gamma, beta, eps=EPS, residual=r, want_stats=True)
    dx, dgamma, dbeta = B.spc_layer_norm_backward(dy, total, mean, rstd, gamma, dsum=e)

    def loss(a, g, b):
        z, _, _, _, y = forward_ref(a, r, g, b, EPS)
        return float((y * dy.double()).sum() + (z * e.double()).sum())

    for t, grad in ((0, dx), (1, dgamma), (2, dbeta)):
        at = [x.double(), gamma.double(), beta.double()]
        d = torch.randn(at[t].shape, generator=gen, dtype=torch.float64).cuda()
        hi, lo, step = list(at), list(at), 1e-4
        hi[t], lo[t] = at[t] + step * d, at[t] - step * d
        num, ana = (loss(*hi) - loss(*lo)) / (2 * step), float((grad.double() * d).sum())
        # (central differences: third derivatives times step^2; fp32 sums of some 1650 terms)
        assert abs(num - ana) <= 1e-5 * float((grad.double() * d).abs().sum()), t


def test_parameters_may_be_missing():
    gen = torch.Generator().manual_seed(4)
    x, dy = rows(100, 48, F32, gen), rows(100, 48, F32, gen)
    one, zero = torch.ones(48, device="cuda"), torch.zeros(48, device="cuda")
    y, s, mean, rstd = B.spc_layer_norm_forward(x)
    assert s is None and mean is None and rstd is None
    assert torch.equal(y, B.spc_layer_norm_forward(x, one, zero)[0])
    _, _, mean, rstd = B.spc_layer_norm_forward(x, want_stats=True)
    a, b = B.spc_layer_norm_backward(dy, x, mean, rstd), B.spc_layer_norm_backward(dy, x, mean, rstd, one)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    dx, dgamma, dbeta = B.spc_layer_norm_backward(dy, x, mean, rstd, want_params=False)
    assert torch.equal(dx, a[0]) and dgamma is None and dbeta is None


@pytest.mark.parametrize("c", [3, 64, 90, 3000, 3001, 7001])
def test_in_place(c):
    gen = torch.Generator().manual_seed(5)
    x, r = rows(300, c, BF16, gen), rows(300, c, BF16, gen)
    y, s, mean, rstd = B.spc_layer_norm_forward(x, residual=r, want_stats=True)
    x2, r2 = x.clone(), r.clone()
    B.spc_layer_norm_forward(x2, residual=r2, out=x2, sum_out=r2)
    assert torch.equal(x2, y) and torch.equal(r2, s)
    dx = B.spc_layer_norm_backward(r, s, mean, rstd, dsum=x)[0]
    r2 = r.clone()
    B.spc_layer_norm_backward(r2, s, mean, rstd, dsum=x, out=r2)
    assert torch.equal(r2, dx)


@pytest.mark.parametrize("c", [24, 64, 90, 1100, 5000])
def test_a_row_that_is_not_finite_stays_alone(c):
    gen = torch.Generator().manual_seed(6)
    x, dy = rows(200, c, F16, gen), rows(200, c, F16, gen)
    y, _, mean, rstd = B.spc_layer_norm_forward(x, want_stats=True)
    dx = B.spc_layer_norm_backward(dy, x, mean, rstd)[0]
    bad = x.clone()
    bad[7, c // 2], bad[100, 0], bad[199, c - 1] = float("inf"), float("nan"), float("-inf")
    keep = torch.ones(200, dtype=torch.bool, device="cuda")
    keep[[7, 100, 199]] = False
    y2, _, mean2, rstd2 = B.spc_layer_norm_forward(bad, want_stats=True)
    assert torch.equal(y2[keep], y[keep]) and y2[~keep].isnan().all()
    assert torch.equal(B.spc_layer_norm_backward(dy, bad, mean2, rstd2)[0][keep], dx[keep])


def test_constant_and_large_rows():
    x = torch.full((5, 96), 3.0, dtype=F16, device="cuda")
    y, _, mean, rstd = B.spc_layer_norm_forward(x, want_stats=True)
    assert (y == 0).all() and (mean == 3).all() and torch.allclose(rstd, torch.full_like(rstd, EPS ** -0.5), rtol=1e-6)
    # a level far above the spread: the differences are exact, sums of squares would not be
    big = (4096 + torch.arange(64, device="cuda", dtype=F32) % 2)[None].repeat(3, 1)
    y = B.spc_layer_norm_forward(big, eps=1e-12)[0]
    assert torch.allclose(y.abs(), torch.ones_like(y), rtol=1e-5)


def test_same_bits_every_time_and_on_another_stream():
    gen = torch.Generator().manual_seed(8)
    x, dy = rows(30_011, 96, F16, gen), rows(30_011, 96, F16, gen)
    _, _, mean, rstd = B.spc_layer_norm_forward(x, want_stats=True)
    first = B.spc_layer_norm_backward(dy, x, mean, rstd)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(other):
            again = B.spc_layer_norm_backward(dy, x, mean, rstd)
        other.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_recorded():
    gen = torch.Generator().manual_seed(9)
    x, dy, gamma = rows(3000, 64, BF16, gen), rows(3000, 64, BF16, gen), (1 + torch.randn(64, generator=gen)).cuda()

    def step():
        y, _, mean, rstd = B.spc_layer_norm_forward(x, gamma, want_stats=True)
        return y, *B.spc_layer_norm_backward(dy, x, mean, rstd, gamma)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = step()
    for _ in range(3):
        x.copy_(rows(3000, 64, BF16, gen))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_rows_far_apart():
    """Row offsets beyond 32 bits."""
    n, pitch, c = 40, 60_000_000, 64
    wide = torch.empty(n * pitch, dtype=F16, device="cuda")
    x = wide.as_strided((n, c), (pitch, 1))
    x.copy_(torch.randn(n, c))
    y, _, mean, rstd = B.spc_layer_norm_forward(x, want_stats=True)
    near = x.clone()
    assert torch.equal(y, B.spc_layer_norm_forward(near)[0])
    assert torch.equal(B.spc_layer_norm_backward(x, x, mean, rstd, out=x)[0], B.spc_layer_norm_backward(near, near, mean, rstd)[0])


def test_refusals():
    x = torch.zeros(4, 8, device="cuda")
    with pytest.raises(B.SpcError) as e:
        B.spc_layer_norm_forward(torch.zeros(1, 8193, device="cuda"))
    assert e.value.code == B.ERR_UNSUPPORTED
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(B.SpcError) as e:
            B.spc_layer_norm_forward(x, eps=eps)
        assert e.value.code == B.ERR_ARG
    with pytest.raises(B.SpcError) as e:
        B.spc_layer_norm_forward(x[:1].expand(4, 8))  # rows on top of each other
    assert e.value.code == B.ERR_ARG
    for call in (lambda: B.spc_layer_norm_forward(x.double()), lambda: B.spc_layer_norm_forward(x.t()), lambda: B.spc_layer_norm_forward(x, x[0, :7].clone()),
                 lambda: B.spc_layer_norm_forward(x, residual=x.half()), lambda: B.spc_layer_norm_forward(x, sum_out=x),
                 lambda: B.spc_layer_norm_backward(x, x, x[:, 0], x[:, 0])):
        with pytest.raises(AssertionError):
            call()
    L = B.lib()
    p = x.data_ptr()
    assert L.spc_layer_norm_forward(p, 8, None, 0, None, None, 1e-5, p, 8, None, 0, None, None, 4, 8, 9, None) == B.ERR_ARG
    assert L.spc_layer_norm_forward(p, 8, p, 8, None, None, 1e-5, p, 8, None, 0, None, None, 4, 8, 2, None) == B.ERR_ARG
    assert L.spc_layer_norm_forward(p, 8, None, 0, None, None, 1e-5, p, 8, None, 0, p, None, 4, 8, 2, None) == B.ERR_ARG
    assert L.spc_layer_norm_forward(p, 7, None, 0, None, None, 1e-5, p, 8, None, 0, None, None, 4, 8, 2, None) == B.ERR_ARG
    assert L.spc_layer_norm_forward(p + 2, 8, None, 0, None, None, 1e-5, p, 8, None, 0, None, None, 3, 8, 2, None) == B.ERR_ARG
    assert L.spc_layer_norm_forward(None, 8, None, 0, None, None, 1e-5, p, 8, None, 0, None, None, 4, 8, 2, None) == B.ERR_ARG
    assert L.spc_layer_norm_forward(p, 8, None, 0, None, None, 1e-5, p, 8, None, 0, None, None, -1, 8, 2, None) == B.ERR_ARG
    assert L.spc_layer_norm_backward(p, 8, p, 8, None, p, None, None, 0, p, 8, None, None, 4, 8, 2, None) == B.ERR_ARG


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("c", [1, 2, 3, 4, 5, 7, 8, 9, 33, 90, 257, 513, 2051])
def test_gradients_of_a_large_mean_with_a_tiny_deviation(c, dtype):
    """mean * rstd leaves the range of 32 bits, (x - mean) * rstd of the row's channels does not: places behind the last channel must not come in.  Values are the
    mean or the next one, so h has no rounding."""
    gen = torch.Generator().manual_seed(c)
    level, rstd = 2.0 ** 90, 2.0 ** 50
    step = level * 2 * U[dtype]
    x = (level + step * torch.randint(0, 2, (20, c), generator=gen)).to(dtype).cuda()
    dy = torch.randn(20, c, generator=gen).to(dtype).cuda()
    gamma = (1 + torch.randn(c, generator=gen)).cuda()
    mean, s = torch.full((20,), level, device="cuda"), torch.full((20,), 1 / step, device="cuda")
    x[10:], s[10:] = level, rstd  # (h of 0 and 1 above, of 0 here)
    dx, dgamma, dbeta = B.spc_layer_norm_backward(dy, x, mean, s, gamma)
    h = (x.double() - level) * s.double()[:, None]
    w = dy.double() * gamma.double()
    ref = s.double()[:, None] * (w - w.mean(1, keepdim=True) - h * (w * h).mean(1, keepdim=True))
    wm, wh = w.abs().mean(1, keepdim=True), (w * h).abs().mean(1, keepdim=True)
    within(dx, ref, U[dtype] * ref.abs() + 2.0 ** -126 + 2.0 ** -16 * s.double()[:, None] * (w.abs() + wm + h.abs() * wh), "dx")
    within(dgamma, (dy.double() * h).sum(0), 2.0 ** -16 * (dy.double() * h).abs().sum(0), "dgamma")
    within(dbeta, dy.double().sum(0), 2.0 ** -16 * dy.double().abs().sum(0), "dbeta")
