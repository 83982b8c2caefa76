"""The block of norms, projections and attention over sorted voxels against the same block in 64 bits.

Tolerances: the largest difference over the largest value.  fp32: five operators in a row, each within some 2^-16 of what it sums up: 1e-4.  16-bit types
round four tensors on the way (fp16 2^-11, bf16 2^-8 each), and a norm's or a projection's sums average such errors: 1e-2 and 6e-2."""
import pytest
import torch

from paper_2511_20834_amd import binding as B
from paper_2511_20834_amd.mixer import VoxelMixer

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
TOL = {F16: 1e-2, BF16: 6e-2, F32: 1e-4}


def block(c, heads, kv_heads, d, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    w_qkv, w_out = r(c, (heads + 2 * kv_heads) * d) * c ** -0.5, r(heads * d, c) * (heads * d) ** -0.5
    decay = -torch.exp2(-3 - 4 * torch.rand(heads, generator=gen))
    p = [1 + 0.2 * r(c), 0.1 * r(c), 1 + 0.2 * r(c), 0.1 * r(c)]
    return VoxelMixer(w_qkv.to(dtype).cuda(), w_out.to(dtype).cuda(), decay.cuda(), *[t.cuda() for t in p], kv_heads=kv_heads)


def cloud(counts, seed):
    """Sorted keys and packing of scenes of so many voxels, in a random order before."""
    gen = torch.Generator().manual_seed(seed)
    rows = []
    for b, n in enumerate(counts):
        lin = torch.randperm(40 ** 3, generator=gen)[:n]
        rows.append(torch.stack([torch.full((n,), b), lin // 1600, lin // 40 % 40, lin % 40], 1))
    rows = torch.cat(rows).to(torch.int32)
    desc = B.spc_pack_desc_fit([0, 0, 0], [39, 39, 39], len(counts), 1, 1)
    keys, perm = B.spc_pack_coords(rows[torch.randperm(len(rows), generator=gen)].cuda(), desc)
    return keys, perm, desc


def reference(m, x, counts, params):
    """z and s in 64 bits, a row at a time (differentiable in x and params)."""
    w_qkv, w_out, g1, b1, g2, b2 = params
    norm = lambda t, g, b: (t - t.mean(1, keepdim=True)) / torch.sqrt(t.var(1, correction=0, keepdim=True) + m.eps) * g + b
    qkv = norm(x, g1, b1) @ w_qkv
    H, G, d = m.heads, m.heads // m.kv_heads, m.d
    q, k, v = [t.unflatten(1, (-1, d)) for t in qkv.split(m.widths, 1)]
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    l = torch.exp(m.log_decay.double().cpu())[:, None, None]
    rows, t = [], 0
    for n in counts:
        S = torch.zeros(H, d, d, dtype=torch.float64)
        for _ in range(n):
            S = l * S + k[t][:, :, None] * v[t][:, None, :]
            rows.append(d ** -0.5 * (q[t][:, :, None] * S).sum(1).flatten())
            t += 1
    s = x + torch.stack(rows) @ w_out
    return norm(s, g2, b2), s


def params64(m):
    return [t.double().cpu().requires_grad_() for t in (m.w_qkv, m.w_out, m.gamma1, m.beta1, m.gamma2, m.beta2)]


def close(got, ref, tol, what):
    got, ref = got.double().cpu(), ref.detach()
    assert got.shape == ref.shape and torch.isfinite(got).all(), what
    err = float((got - ref).abs().max() / ref.abs().max())
    assert err <= tol, (what, err)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("c,heads,kv_heads,d", [(64, 4, 4, 16), (48, 4, 2, 24), (32, 1, 1, 32)])
def test_forward_and_backward(c, heads, kv_heads, d, dtype):
    counts = [150, 0, 200]
    m = block(c, heads, kv_heads, d, dtype, 3)
    keys, perm, desc = cloud(counts, 4)
    gen = torch.Generator().manual_seed(5)
    x = B.spc_permute_rows(torch.randn(350, c, generator=gen).to(dtype).cuda(), perm)
    dz, ds = (torch.randn(350, c, generator=gen).to(dtype).cuda() for _ in range(2))
    kmap, offsets = m.scenes(keys, desc, 3)
    assert offsets.tolist() == [0, 150, 150, 350]
    z, s, saved = m.forward(x, kmap, offsets, save=True)
    p = params64(m)
    x64 = x.double().cpu().requires_grad_()
    rz, rs = reference(m, x64, counts, p)
    close(z, rz, TOL[dtype], "z")
    close(s, rs, TOL[dtype], "s")
    assert all(torch.equal(a, b) for a, b in zip(m.forward(x, kmap, offsets), (z, s)))
    got = m.backward(dz, ds, saved)
    grads = torch.autograd.grad((rz * dz.double().cpu()).sum() + (rs * ds.double().cpu()).sum(), [x64, *p])
    ref = dict(zip(("x", "w_qkv", "w_out", "gamma1", "beta1", "gamma2", "beta2"), grads))
    for name in got._fields:
        close(getattr(got, name), ref[name], TOL[dtype], name)


def test_streams_give_the_scene_row_by_row():
    m = block(64, 4, 2, 16, F32, 7)
    keys, _, desc = cloud([120, 120], 8)
    x = torch.randn(240, 64, generator=torch.Generator().manual_seed(9)).cuda()
    kmap, offsets = m.scenes(keys, desc, 2)
    z, s = m.forward(x, kmap, offsets)
    state, rows = m.begin(2)
    for t in range(120):
        zt, st = m.step(x[[t, 120 + t]], state, rows)
        close(zt, z[[t, 120 + t]].double().cpu(), TOL[F32], t)
        close(st, s[[t, 120 + t]].double().cpu(), TOL[F32], t)


def test_recorded():
    m = block(64, 4, 4, 16, F16, 11)
    keys, perm, desc = cloud([700, 500], 12)
    kmap, offsets = m.scenes(keys, desc, 2)
    x, dz = torch.randn(1200, 64, device="cuda").half(), torch.randn(1200, 64, device="cuda").half()

    def step():
        z, s, saved = m.forward(x, kmap, offsets, save=True)
        g = m.backward(dz, None, saved)
        return z, s, g.x, g.gamma1, g.beta2  # (the weights' products are a library's)

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


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (4, 2)])
@pytest.mark.parametrize("rejected", [0, 1, 70])
def test_rows_in_no_scene_stay_out(rejected, heads, kv_heads, dtype):
    """Rejected rows lie behind the last scene.  They hold NaN in every input, and the memory that buffers are taken from is full of NaN: results of the other rows
    and all gradients are those of the other rows alone."""
    counts, c, d = [150, 0, 200], 64, 16
    m = block(c, heads, kv_heads, d, dtype, 13)
    gen = torch.Generator().manual_seed(14)
    rows = []
    for b, n in enumerate(counts):
        lin = torch.randperm(40 ** 3, generator=gen)[:n]
        rows.append(torch.stack([torch.full((n,), b), lin // 1600, lin // 40 % 40, lin % 40], 1))
    rows = torch.cat([*rows, torch.full((rejected, 4), 1000)]).to(torch.int32).cuda()
    n = 350 + rejected
    desc = B.spc_pack_desc_fit([0, 0, 0], [39, 39, 39], 3, 1, 1)
    keys, perm = B.spc_pack_coords(rows, desc)
    kmap, offsets = m.scenes(keys, desc, 3)
    assert offsets.tolist() == [0, 150, 150, 350]
    x, dz, ds = (torch.randn(n, c, generator=gen).to(dtype).cuda() for _ in range(3))
    for t in (x, dz, ds):
        t[350:] = float("nan")
    stale = [torch.full((n, w), float("nan"), dtype=t, device="cuda") for t in (dtype, torch.float32) for w in (1, c, heads * d, (heads + 2 * kv_heads) * d) for _ in range(8)]
    del stale
    z, s, saved = m.forward(x, kmap, offsets, save=True)
    got = m.backward(dz, ds, saved)
    p = params64(m)
    x64 = x[:350].double().cpu().requires_grad_()
    rz, rs = reference(m, x64, counts, p)
    close(z[:350], rz, TOL[dtype], "z")
    close(s[:350], rs, TOL[dtype], "s")
    assert all(torch.equal(a[:350], b[:350]) for a, b in zip(m.forward(x, kmap, offsets), (z, s)))
    grads = torch.autograd.grad((rz * dz[:350].double().cpu()).sum() + (rs * ds[:350].double().cpu()).sum(), [x64, *p])
    ref = dict(zip(("x", "w_qkv", "w_out", "gamma1", "beta1", "gamma2", "beta2"), grads))
    assert (got.x[350:] == 0).all()
    for name in got._fields:
        close(getattr(got, name)[:350] if name == "x" else getattr(got, name), ref[name], TOL[dtype], name)


def test_scenes_in_the_middle_of_the_rows():
    """Offsets of a part of the rows, in front and behind as well; without a second gradient."""
    m = block(32, 2, 1, 16, F32, 15)
    keys, _, desc = cloud([90, 60, 50], 16)
    gen = torch.Generator().manual_seed(17)
    x, dz = (torch.randn(200, 32, generator=gen).cuda() for _ in range(2))
    kmap, offsets = m.scenes(keys, desc, 3)
    x[:90], x[150:], dz[:90], dz[150:] = float("nan"), float("inf"), float("nan"), float("inf")
    z, s, saved = m.forward(x, kmap, offsets[1:3].contiguous(), save=True)
    got = m.backward(dz, None, saved)
    p = params64(m)
    x64 = x[90:150].double().cpu().requires_grad_()
    rz, _ = reference(m, x64, [60], p)
    close(z[90:150], rz, TOL[F32], "z")
    grads = torch.autograd.grad((rz * dz[90:150].double().cpu()).sum(), [x64, *p])
    ref = dict(zip(("x", "w_qkv", "w_out", "gamma1", "beta1", "gamma2", "beta2"), grads))
    assert (got.x[:90] == 0).all() and (got.x[150:] == 0).all()
    for name in got._fields:
        close(getattr(got, name)[90:150] if name == "x" else getattr(got, name), ref[name], TOL[F32], name)


def test_all_rows_said_to_lie_in_scenes():
    """The same bits where that is so."""
    m = block(64, 4, 2, 16, BF16, 18)
    keys, _, desc = cloud([150, 0, 200], 19)
    x, dz, ds = (torch.randn(350, 64, generator=torch.Generator().manual_seed(20 + i)).to(BF16).cuda() for i in range(3))
    kmap, offsets = m.scenes(keys, desc, 3)
    z, s, saved = m.forward(x, kmap, offsets, save=True)
    z2, s2, saved2 = m.forward(x, kmap, offsets, save=True, all_rows=True)
    assert torch.equal(z, z2) and torch.equal(s, s2)
    assert all(torch.equal(a, b) for a, b in zip(m.backward(dz, ds, saved), m.backward(dz, ds, saved2)))
