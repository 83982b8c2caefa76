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
