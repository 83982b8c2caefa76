"""Root-mean-square norm of feature rows (16, 32 and 8-bit outputs, gradients), rows in 8 bits and their product, against the formulas in 64 bits.

Tolerances.  u is half a unit in the last place of the rows' type (2^-11 fp16, 2^-8 bf16, 2^-24 fp32): the one rounding of an output.  Sums of
a row are trees of at most 32 + 8 fp32 additions of squares: 2^-18 of the sum, half of that of rstd.  A column sum is a chain of at most some 200
additions for the sizes here, 2^-16 of the sum of magnitudes.  An e4m3 value is off by half a step: 2^-4 of itself from 2^-6 on, 2^-10 below."""
import pytest
import torch

from paper_2511_20834_amd import binding as B

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
F8 = torch.float8_e4m3fn
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
    assert got.shape == ref.shape, what
    if not got.numel():
        return
    over = (got - ref.cpu()).abs() - tol
    assert torch.isfinite(got).all() and over.max() <= 0, (what, float(over.max()), int(over.argmax()))


def reference(x, r, gamma):
    z = x.double() if r is None else x.double() + r.double()
    rstd = (z.square().mean(1) + EPS) ** -0.5
    h = z * rstd[:, None]
    return z, rstd, h, h if gamma is None else h * gamma.double()


def check_bytes(q, scale, y, lost, what):
    """q scale is y rounded to 8 bits: values behind the scale are off by `lost` of themselves before that."""
    top = y.abs().amax(1).clamp(min=2.0 ** -100)
    s = scale.double()
    within(scale, top / 448, 2 * lost * top / 448, what + " scale")
    got = q.double() * s[:, None]
    step = torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * s[:, None])
    within(got, y, step * (1 + 4 * lost) + 4 * lost * y.abs(), what)


SHAPES = [(1, 1), (3, 2), (1, 64), (257, 5), (33, 90), (700, 16), (129, 24), (65, 100), (1000, 64), (77, 257), (40, 512), (31, 513), (9, 1024), (5, 2048),
          (6, 2050), (3, 2051), (4, 4099), (2, 8192), (3, 8191)]
LAYOUTS = [(False, 0, 0), (True, 8, 0), (True, 1, 1), (False, 6, 2)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("extra,pitch,first", LAYOUTS)
def test_forward(n, c, dtype, extra, pitch, first):
    gen = torch.Generator().manual_seed(n * 10007 + c)
    p = c + pitch if pitch else 0
    x, r = rows(n, c, dtype, gen, p, first), rows(n, c, dtype, gen, p, first) if extra else None
    gamma = (1 + torch.randn(c, generator=gen)).cuda()
    out = torch.full((n, c + pitch + 3), 7.0, dtype=dtype, device="cuda")
    y, s, rstd = B.spc_rms_norm_forward(x, gamma, eps=EPS, residual=r, want_stats=True, out=out[:, first:first + c])
    z, rs, _, ref = reference(x, r, gamma)
    within(rstd, rs, 2.0 ** -18 * rs, "rstd")
    within(y, ref, (U[dtype] + 2.0 ** -17) * ref.abs() + TINY[dtype], "y")
    if extra:
        within(s, z, (U[dtype] + 2.0 ** -23) * z.abs() + TINY[dtype], "sum")
    else:
        assert s is None
    assert (out[:, :first] == 7).all() and (out[:, first + c:] == 7).all()
    # the same in 8 bits
    wide = torch.full((n, c + pitch + 3), 7.0, device="cuda").to(F8)
    q, scale, s8, rstd8 = B.spc_rms_norm_quantize(x, gamma, eps=EPS, residual=r, want_stats=True, out=wide[:, first:first + c])
    check_bytes(q, scale, ref, 2.0 ** -17, "q")
    assert torch.equal(rstd8, rstd) and (s8 is None if r is None else torch.equal(s8, s))
    assert (wide[:, :first].float() == 7).all() and (wide[:, first + c:].float() == 7).all()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("n,c", SHAPES + [(0, 64), (6011, 128), (20_000, 36)])
@pytest.mark.parametrize("extra,pitch,first", LAYOUTS)
def test_backward(n, c, dtype, extra, pitch, first):
    gen = torch.Generator().manual_seed(n * 10007 + c + 1)
    p = c + pitch if pitch else 0
    x, dy, e = rows(n, c, dtype, gen, p, first), rows(n, c, dtype, gen, p, first), rows(n, c, dtype, gen, p, first) if extra else None
    gamma = (1 + torch.randn(c, generator=gen)).cuda()
    rstd = reference(x, None, None)[1].float()
    dx, dgamma = B.spc_rms_norm_backward(dy, x, rstd, gamma, dsum=e)
    s = rstd.double()[:, None]
    h, w = x.double() * s, dy.double() * gamma.double()
    ref = s * (w - h * (w * h).mean(1, keepdim=True)) + (e.double() if extra else 0.0)
    lost = 2.0 ** -17 * s * (w.abs() + h.abs() * (w * h).abs().mean(1, keepdim=True))
    within(dx, ref, (U[dtype] + 2.0 ** -23) * ref.abs() + TINY[dtype] + lost, "dx")
    within(dgamma, (dy.double() * h).sum(0), 2.0 ** -16 * (dy.double() * h).abs().sum(0), "dgamma")


def test_gradients_against_differences():
    """The fp32 backward pass along random directions against central differences of the forward pass in 64 bits."""
    gen = torch.Generator().manual_seed(3)
    n, c = 50, 33
    x, r, dy, e = (rows(n, c, F32, gen) for _ in range(4))
    gamma = (1 + torch.randn(c, generator=gen)).cuda()
    _, total, rstd = B.spc_rms_norm_forward(x, gamma, eps=EPS, residual=r, want_stats=True)
    dx, dgamma = B.spc_rms_norm_backward(dy, total, rstd, gamma, dsum=e)

    def loss(a, g):
        z, _, _, y = reference(a, r, g)
        return float((y * dy.double()).sum() + (z * e.double()).sum())

    for t, grad in ((0, dx), (1, dgamma)):
        at = [x.double(), gamma.double()]
        d = torch.randn(at[t].shape, generator=gen, dtype=torch.float64).cuda()
        hi, lo, step = list(at), list(at), 1e-4
        hi[t], lo[t] = at[t] + step * d, at[t] - step * d
        num, ana = (loss(*hi) - loss(*lo)) / (2 * step), float((grad.double() * d).sum())
        # (central differences: third derivatives times step^2; fp32 sums of some 1650 terms)
        assert abs(num - ana) <= 1e-5 * float((grad.double() * d).abs().sum()), t


def test_parameters_may_be_missing():
    gen = torch.Generator().manual_seed(4)
    x, dy, one = rows(100, 48, F32, gen), rows(100, 48, F32, gen), torch.ones(48, device="cuda")
    y, s, rstd = B.spc_rms_norm_forward(x)
    assert s is None and rstd is None
    assert torch.equal(y, B.spc_rms_norm_forward(x, one)[0])
    a, b = B.spc_rms_norm_quantize(x), B.spc_rms_norm_quantize(x, one)
    assert torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8)) and torch.equal(a[1], b[1]) and a[2] is None and a[3] is None
    rstd = B.spc_rms_norm_forward(x, want_stats=True)[2]
    assert all(torch.equal(p, q) for p, q in zip(B.spc_rms_norm_backward(dy, x, rstd), B.spc_rms_norm_backward(dy, x, rstd, one)))
    dx, dgamma = B.spc_rms_norm_backward(dy, x, rstd, want_params=False)
    assert torch.equal(dx, B.spc_rms_norm_backward(dy, x, rstd)[0]) and dgamma is None


@pytest.mark.parametrize("c", [3, 64, 90, 3000, 3001, 7001])
def test_in_place(c):
    gen = torch.Generator().manual_seed(5)
    x, r = rows(300, c, BF16, gen), rows(300, c, BF16, gen)
    y, s, rstd = B.spc_rms_norm_forward(x, residual=r, want_stats=True)
    x2, r2 = x.clone(), r.clone()
    B.spc_rms_norm_forward(x2, residual=r2, out=x2, sum_out=r2)
    assert torch.equal(x2, y) and torch.equal(r2, s)
    q, scale, _, _ = B.spc_rms_norm_quantize(x, residual=r)
    r2 = r.clone()
    q2, scale2, _, _ = B.spc_rms_norm_quantize(x, residual=r2, sum_out=r2)
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(scale, scale2) and torch.equal(r2, s)
    dx = B.spc_rms_norm_backward(r, s, rstd, dsum=x)[0]
    for at in range(3):
        t = [r.clone(), s.clone(), x.clone()]
        B.spc_rms_norm_backward(t[0], t[1], rstd, dsum=t[2], out=t[at])
        assert torch.equal(t[at], dx), at


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("c", [1, 7, 8, 64, 90, 1000, 5000])
def test_rows_in_8_bits(c, dtype):
    """Bit for bit: the largest value, 448 over it and the products are single roundings."""
    gen = torch.Generator().manual_seed(6 + c)
    x = (torch.randn(70, c, generator=gen) * torch.exp2(40 * torch.rand(70, 1, generator=gen) - 20 if dtype != F16 else 8 * torch.rand(70, 1, generator=gen) - 4)).to(dtype).cuda()
    x[5] = 0
    q, scale = B.spc_quantize_rows(x)
    top = x.float().abs().amax(1).clamp(min=2.0 ** -100)
    # (quotients in 64 bits, rounded once more, are those of 32 bits; torch's own by a number are products with its reciprocal)
    assert torch.equal(scale, (top.double() / 448).float())
    up = (448 / top.double()).float()
    assert torch.equal(q.view(torch.uint8), (x.float() * up[:, None]).to(F8).view(torch.uint8))
    assert (q[5].float() == 0).all() and torch.isfinite(q.float()).all()


def test_infinities_and_nan_stay_in_their_rows():
    gen = torch.Generator().manual_seed(7)
    x, dy, g = rows(40, 90, F32, gen), rows(40, 90, F32, gen), torch.ones(90, device="cuda")
    y, _, rstd = B.spc_rms_norm_forward(x, g, want_stats=True)
    q, scale, _, _ = B.spc_rms_norm_quantize(x, g)
    bad = x.clone()
    bad[3, 4], bad[7, 89], bad[11] = float("nan"), float("inf"), -float("inf")
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[3, 7, 11]] = False
    y2, _, rstd2 = B.spc_rms_norm_forward(bad, g, want_stats=True)
    q2, scale2, _, _ = B.spc_rms_norm_quantize(bad, g)
    assert torch.equal(y2[keep], y[keep]) and torch.equal(rstd2[keep], rstd[keep]) and torch.equal(scale2[keep], scale[keep])
    assert torch.equal(q2[keep].view(torch.uint8), q[keep].view(torch.uint8))
    assert torch.isnan(y2[3]).all() and torch.isnan(y2[7, 89]) and torch.isnan(q2[3].float()).all() and torch.isnan(q2[11].float()).all()
    dx, _ = B.spc_rms_norm_backward(dy, x, rstd, g)
    assert torch.equal(B.spc_rms_norm_backward(dy, bad, rstd, g)[0][keep], dx[keep])
    plain, plain_scale = B.spc_quantize_rows(bad)
    assert torch.isnan(plain[3, 4].float()) and torch.isinf(plain_scale[7]) and torch.isfinite(plain_scale[3])


# ---------------------------------------------------------------- products
def operand(n, c, gen, pitch=0, first=0):
    q, scale = B.spc_quantize_rows(torch.randn(n, c, generator=gen).cuda())
    if not pitch:
        return q, scale
    wide = torch.full((n, c + pitch), float("nan"), device="cuda").to(F8)
    wide[:, first:first + c] = q
    return wide[:, first:first + c], scale


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("n,c,m", [(1, 1, 1), (1, 16, 32), (5, 7, 3), (130, 64, 64), (129, 128, 65), (300, 100, 200), (64, 129, 130), (257, 256, 512), (40, 300, 90), (33, 512, 17), (70, 513, 100),
                                   (20, 1500, 48), (2000, 48, 24), (127, 255, 1000)])
@pytest.mark.parametrize("pitch,first", [(0, 0), (5, 3)])
def test_product(n, c, m, dtype, pitch, first):
    """Every addition may be off by a unit in the last place (2^-23) of the sum of magnitudes, the scales' products by 2^-22."""
    gen = torch.Generator().manual_seed(n + 31 * c + 1009 * m)
    (x, sx), (w, sw) = operand(n, c, gen, pitch, first), operand(m, c, gen, pitch, first)
    out = torch.full((n, m + pitch + 2), 7.0, dtype=dtype, device="cuda")
    y = B.spc_linear_f8(x, sx, w, sw, out=out[:, first:first + m])
    a, b = x.double() * sx.double()[:, None], w.double() * sw.double()[:, None]
    ref, mag = a @ b.t().contiguous(), a.abs() @ b.abs().t().contiguous()
    within(y, ref, (U[dtype] + 2.0 ** -22) * ref.abs() + TINY[dtype] + c * 2.0 ** -23 * mag, "y")
    assert (out[:, :first] == 7).all() and (out[:, first + m:] == 7).all()
    assert torch.equal(y, B.spc_linear_f8(x.contiguous(), sx, w.contiguous(), sw, dtype=dtype))


def test_product_keeps_nan_to_its_row_and_column():
    gen = torch.Generator().manual_seed(8)
    (x, sx), (w, sw) = operand(200, 100, gen), operand(150, 100, gen)
    y = B.spc_linear_f8(x, sx, w, sw, dtype=F32)
    nan = torch.full((1,), float("nan"), device="cuda").to(F8)
    x, w = x.clone(), w.clone()
    x[77, 99], w[33, 0] = nan[0], nan[0]
    z = B.spc_linear_f8(x, sx, w, sw, dtype=F32)
    bad = torch.isnan(z)
    assert bad[77].all() and bad[:, 33].all() and int(bad.sum()) == 200 + 150 - 1
    assert torch.equal(z[~bad], y[~bad])


def test_norm_and_product_recorded():
    """A served block's front in a graph: norm to 8 bits, product; and the gradients' calls."""
    gen = torch.Generator().manual_seed(9)
    x, r, dy = (rows(3000, 128, BF16, gen) for _ in range(3))
    w, sw = operand(256, 128, gen)
    g = torch.ones(128, device="cuda")

    def step():
        q, scale, s, rstd = B.spc_rms_norm_quantize(x, g, residual=r, want_stats=True)
        return (B.spc_linear_f8(q, scale, w, sw), s, *B.spc_rms_norm_backward(dy, s, rstd, g, dsum=x))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for _ in range(3):
        x.normal_()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("c", [1, 3, 64, 90, 257, 1024, 2051, 8192])
@pytest.mark.parametrize("extra", [False, True])
def test_rows_of_large_values(extra, c, dtype):
    """Rows of 2^50 to 2^124, whose squares add up beyond 32 bits: tolerances as everywhere, with the type's spacing near zero where rstd and its products are as small."""
    gen = torch.Generator().manual_seed(c)
    size = 2.0 ** torch.arange(50, 125, dtype=torch.float64)[:, None]
    big = lambda: (torch.randn(75, c, generator=gen).clamp(-4, 4) * size).to(dtype).cuda()  # noqa: E731
    x, r, dy = big(), big() if extra else None, rows(75, c, dtype, gen)
    gamma = (1 + torch.randn(c, generator=gen)).cuda()
    y, s, rstd = B.spc_rms_norm_forward(x, gamma, eps=EPS, residual=r, want_stats=True)
    z, rs, h, ref = reference(x, r, gamma)
    near = {BF16: 2.0 ** -133, F32: 2.0 ** -149}[dtype]
    within(rstd, rs, 2.0 ** -18 * rs + 2.0 ** -149, "rstd")
    within(y, ref, (U[dtype] + 2.0 ** -17) * ref.abs(), "y")
    q, scale, s8, rstd8 = B.spc_rms_norm_quantize(x, gamma, eps=EPS, residual=r, want_stats=True)
    check_bytes(q, scale, ref, 2.0 ** -17, "q")
    assert torch.equal(rstd8, rstd) and (s8 is None if r is None else torch.equal(s8, s))
    x = x if s is None else s
    dx, dgamma = B.spc_rms_norm_backward(dy, x, rstd, gamma)
    k = rstd.double()[:, None]
    h, w = x.double() * k, dy.double() * gamma.double()
    ref = k * (w - h * (w * h).mean(1, keepdim=True))
    lost = 2.0 ** -17 * k * (w.abs() + h.abs() * (w * h).abs().mean(1, keepdim=True))
    within(dx, ref, (U[dtype] + 2.0 ** -23) * ref.abs() + near + lost, "dx")
    within(dgamma, (dy.double() * h).sum(0), 2.0 ** -16 * (dy.double() * h).abs().sum(0), "dgamma")
