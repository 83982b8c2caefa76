"""The selective state space block over sorted voxels against the same block in 64 bits.

Tolerances: the largest difference over the largest value.  fp32: eight operators in a row, each within some 2^-16 of what it sums up: 1e-4.  16-bit types round seven tensors on
the way (fp16 2^-11, bf16 2^-8 each), whose errors the sums behind them average: 1e-2 and 6e-2. 

8 bits, by the 2-norm: an e4m3 value is off by up to 2^-4 of itself, evenly spread over a step that is 2^-3 to 2^-4 of it: 2.6 % (2-norm).  The first projection's products have
two such errors, independent from term to term: 3.7 % of its outputs.  The result is a product of four of these (u, B and C, which are made of u, and the gate), the steps' share
aside: 3.7 % times 2 if they were independent, times 4 if they went together: 15 %."""
import pytest
import torch

from paper_2511_20834_amd import binding as B
from paper_2511_20834_amd.scanner import VoxelScan

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
TOL = {F16: 1e-2, BF16: 6e-2, F32: 1e-4}
NAMES = ("x", "gamma", "w_in", "conv_weight", "conv_bias", "w_x", "w_dt", "dt_bias", "A", "skip", "w_out")


def block(c, d, N, rank, width, groups, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    w = lambda i, o: (r(i, o) * i ** -0.5).to(dtype).cuda()  # noqa: E731
    step = torch.exp(torch.rand(d, generator=gen) * 4.6 - 6.9)
    return VoxelScan((1 + 0.2 * r(c)).cuda(), w(c, 2 * d), (r(d, width) * width ** -0.5).cuda(), (0.1 * r(d)).cuda(), w(d, rank + 2 * groups * N), w(rank, d),
                     (step + torch.log(-torch.expm1(-step))).cuda(), (-torch.arange(1, N + 1) * torch.exp(0.1 * r(d, N))).cuda(), (1 + 0.2 * r(d)).cuda(), w(d, c), groups=groups)


def cloud(counts, seed, rejected=0):
    """Sorted keys and packing of scenes of so many voxels, in a random order before."""
    gen = torch.Generator().manual_seed(seed)
    rows = []
    for b, n in enumerate(counts):
        lin = torch.randperm(40 ** 3, generator=gen)[:n]
        rows.append(torch.stack([torch.full((n,), b), lin // 1600, lin // 40 % 40, lin % 40], 1))
    rows = torch.cat([*rows, torch.full((rejected, 4), 1000)]).to(torch.int32)
    desc = B.spc_pack_desc_fit([0, 0, 0], [39, 39, 39], len(counts), 1, 1)
    keys, _ = B.spc_pack_coords(rows.cuda(), desc)
    return keys, desc


def params64(m):
    return [getattr(m, n).double().cpu().requires_grad_() for n in NAMES[1:]]


def reference(m, x, counts, params):
    """result and s in 64 bits, a row at a time (differentiable in x and params); x with the residual added."""
    gamma, w_in, conv_w, conv_b, w_x, w_dt, dt_bias, A, skip, w_out = params
    silu = torch.nn.functional.silu
    y = x * (x.square().mean(1, keepdim=True) + m.eps) ** -0.5 * gamma
    u, z = (y @ w_in).split(m.d, 1)
    parts, at = [], 0
    for n in counts:
        seq = torch.cat([torch.zeros(m.width - 1, m.d, dtype=torch.float64), u[at:at + n]])
        parts.append(conv_b + sum(conv_w[:, j] * seq[j:j + n] for j in range(m.width)))
        at += n
    u = silu(torch.cat(parts))
    t, b, c = (u @ w_x).split(m.widths, 1)
    wide = lambda v: v.unflatten(1, (m.groups, m.states)).repeat_interleave(m.d // m.groups, 1)  # noqa: E731
    b, c = wide(b), wide(c)
    delta = torch.nn.functional.softplus(t @ w_dt + dt_bias)
    rows, at = [], 0
    for n in counts:
        h = torch.zeros(m.d, m.states, dtype=torch.float64)
        for i in range(at, at + n):
            h = torch.exp(delta[i][:, None] * A) * h + (delta[i] * u[i])[:, None] * b[i]
            rows.append((h * c[i]).sum(1) + skip * u[i])
        at += n
    return (torch.stack(rows) * silu(z)) @ w_out, x


def close(got, ref, tol, what):
    got, ref = got.double().cpu(), ref.detach()
    assert got.shape == ref.shape and torch.isfinite(got).all(), what
    err = float((got - ref).abs().max() / ref.abs().max())
    assert err <= tol, (what, err)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("c,d,N,rank,width,groups", [(64, 128, 16, 8, 4, 1), (48, 90, 8, 5, 3, 2), (32, 64, 4, 16, 2, 1)])
@pytest.mark.parametrize("residual", [False, True])
def test_forward_and_backward(c, d, N, rank, width, groups, residual, dtype):
    counts = [90, 0, 110]
    m = block(c, d, N, rank, width, groups, dtype, 3)
    keys, desc = cloud(counts, 4)
    gen = torch.Generator().manual_seed(5)
    x, r, dout, ds = (torch.randn(200, c, generator=gen).to(dtype).cuda() for _ in range(4))
    r = r if residual else None
    kmap, offsets = m.scenes(keys, desc, 3)
    out, s, saved = m.forward(x, kmap, offsets, r, save=True)
    p = params64(m)
    x64 = (x.double() + (r.double() if residual else 0)).cpu().requires_grad_()
    ro, rs = reference(m, x64, counts, p)
    close(out, ro, TOL[dtype], "result")
    close(s, rs, TOL[dtype], "s")
    assert all(torch.equal(a, b) for a, b in zip(m.forward(x, kmap, offsets, r), (out, s)))
    assert all(torch.equal(a, b) for a, b in zip(m.forward(x, kmap, offsets, r, save=True, all_rows=True)[:2], (out, s)))
    for with_sum in (True, False):
        got = m.backward(dout, ds if with_sum else None, saved)
        loss = (ro * dout.double().cpu()).sum() + ((rs * ds.double().cpu()).sum() if with_sum else 0)
        ref = dict(zip(NAMES, torch.autograd.grad(loss, [x64, *p], retain_graph=True)))
        for name in got._fields:
            close(getattr(got, name), ref[name], TOL[dtype], name)


def test_streams_give_the_scene_row_by_row():
    m = block(64, 96, 16, 8, 4, 2, F32, 7)
    keys, desc = cloud([120, 120], 8)
    x, r = (torch.randn(240, 64, generator=torch.Generator().manual_seed(9 + i)).cuda() for i in range(2))
    kmap, offsets = m.scenes(keys, desc, 2)
    out, s = m.forward(x, kmap, offsets, r)
    state, rows = m.begin(2)
    for t in range(120):
        ot, st = m.step(x[[t, 120 + t]], state, rows, r[[t, 120 + t]])
        close(ot, out[[t, 120 + t]].double().cpu(), TOL[F32], t)
        close(st, s[[t, 120 + t]].double().cpu(), TOL[F32], t)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("c,d", [(64, 128), (90, 100)])
def test_served_in_8_bits(c, d, dtype):
    m = block(c, d, 16, 8, 4, 1, dtype, 10)
    e = m.in_8_bits()
    keys, desc = cloud([150, 50], 11)
    x, r = (torch.randn(200, c, generator=torch.Generator().manual_seed(12 + i)).to(dtype).cuda() for i in range(2))
    kmap, offsets = m.scenes(keys, desc, 2)
    out, s = m.forward(x, kmap, offsets, r)
    out8, s8 = e.forward(x, kmap, offsets, r)
    assert torch.equal(s, s8)
    assert float((out8.double() - out.double()).norm() / out.double().norm()) <= 0.15
    state, rows = e.begin(2)
    for t in range(50):  # (one row of each scene at a time)
        ot, _ = e.step(x[[t, 150 + t]], state, rows, r[[t, 150 + t]])
        assert (ot - out8[[t, 150 + t]]).abs().max() <= TOL[dtype] * out8.abs().max()
    with pytest.raises(AssertionError):
        e.forward(x, kmap, offsets, r, save=True)


def test_recorded():
    m = block(64, 128, 16, 8, 4, 1, F16, 13)
    keys, desc = cloud([700, 500], 14)
    kmap, offsets = m.scenes(keys, desc, 2)
    x, dout = torch.randn(1200, 64, device="cuda").half(), torch.randn(1200, 64, device="cuda").half()

    def step():
        out, s, saved = m.forward(x, kmap, offsets, save=True)
        g = m.backward(dout, None, saved)
        return out, s, g.x, g.gamma, g.conv_weight, g.A, g.dt_bias, g.skip  # (the weights' products are a library's)

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


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("rejected", [1, 70])
def test_rows_in_no_scene_stay_out(rejected, dtype):
    """Rejected rows lie behind the last scene.  They hold NaN in every input, and the memory that buffers are taken from is full of NaN: results of the other rows
    and all gradients are those of the other rows alone."""
    counts, c, d = [100, 0, 80], 64, 70
    m = block(c, d, 8, 8, 4, 1, dtype, 15)
    keys, desc = cloud(counts, 16, rejected)
    kmap, offsets = m.scenes(keys, desc, 3)
    assert offsets.tolist() == [0, 100, 100, 180]
    gen = torch.Generator().manual_seed(17)
    n = 180 + rejected
    x, r, dout, ds = (torch.randn(n, c, generator=gen).to(dtype).cuda() for _ in range(4))
    for t in (x, r, dout, ds):
        t[180:] = float("nan")
    stale = [torch.full((n, w), float("nan"), dtype=t, device="cuda") for t in (dtype, F32) for w in (1, c, d, 2 * d, 24) for _ in range(8)]
    del stale
    out, s, saved = m.forward(x, kmap, offsets, r, save=True)
    got = m.backward(dout, ds, saved)
    p = params64(m)
    x64 = (x.double() + r.double())[:180].cpu().requires_grad_()
    ro, rs = reference(m, x64, counts, p)
    close(out[:180], ro, TOL[dtype], "result")
    close(s[:180], rs, TOL[dtype], "s")
    assert all(torch.equal(a[:180], b[:180]) for a, b in zip(m.forward(x, kmap, offsets, r), (out, s)))
    grads = torch.autograd.grad((ro * dout[:180].double().cpu()).sum() + (rs * ds[:180].double().cpu()).sum(), [x64, *p])
    ref = dict(zip(NAMES, grads))
    assert (got.x[180:] == 0).all()
    for name in got._fields:
        close(getattr(got, name)[:180] if name == "x" else getattr(got, name), ref[name], TOL[dtype], name)
