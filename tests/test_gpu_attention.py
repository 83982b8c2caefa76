"""Linear attention with decays, forward, backward and a row at a time, against its recurrence in 64 bits.

Tolerances.  An output is rounded once to its type (u: half a unit in the last place), and is a sum of products whose magnitudes add up to what the same
recurrence gives for absolute values, B.  fp32 chains here have some 64 + 128 + 128 links and factors of decays are good to a few 2^-24: 2^-16 of
B.  16-bit types take sums that pass through the matrix units as two pieces of at least 8 bits each, 2^-16 of B once more on either side."""
import itertools

import pytest
import torch

from paper_2511_20834_amd import binding as B

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
U = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}
TINY = {F16: 2.0 ** -24, BF16: 2.0 ** -126, F32: 2.0 ** -126}  # spacing of fp16 near zero, smallest normal numbers
PART = {F16: 2.0 ** -14, BF16: 2.0 ** -14, F32: 2.0 ** -16}


def recur(q, k, v, g, at, scale, S0=None):
    """(out, last states) in 64 bits, a row at a time (differentiable)."""
    H, G = q.shape[1], q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    l = torch.exp(g)[:, None, None]
    out, last = [torch.zeros(0, H, v.shape[2], dtype=torch.float64)], []
    for b in range(len(at) - 1):
        S = torch.zeros(H, q.shape[2], v.shape[2], dtype=torch.float64) if S0 is None else S0[b]
        for t in range(at[b], at[b + 1]):
            S = torch.where(l > 0, l * S, 0.0) + k[t][:, :, None] * v[t][:, None, :]
            out.append(scale * (q[t][:, :, None] * S).sum(1)[None])
        last.append(S)
    return torch.cat(out), torch.stack(last)


def make(lengths, heads, kv, dk, dv, dtype, seed, states, decay=None, layout="columns"):
    gen = torch.Generator().manual_seed(seed)
    n = sum(lengths)
    qkv = torch.randn(n, heads * dk + kv * (dk + dv), generator=gen).to(dtype).cuda()
    q, k, v = qkv.split([heads * dk, kv * dk, kv * dv], 1)
    q, k, v = q.unflatten(1, (heads, dk)), k.unflatten(1, (kv, dk)), v.unflatten(1, (kv, dv))
    if layout == "heads":  # [heads, rows, channels] in memory
        q, k, v = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v))
    elif layout == "rows":
        q, k, v = (t.contiguous() for t in (q, k, v))
    g = -torch.exp2(-1 - 8 * torch.rand(heads, generator=gen)) if decay is None else torch.full((heads,), decay)
    at = [0] + list(itertools.accumulate(lengths))
    S0 = torch.randn(len(lengths), heads, dk, dv, generator=gen).cuda() if states else None
    return q, k, v, g.cuda(), torch.tensor(at, dtype=torch.int32).cuda(), at, S0


def cpu(t):
    return None if t is None else t.detach().double().cpu()


def within(got, ref, mag, dtype, what):
    got = cpu(got)
    u, tiny = (U[dtype], TINY[dtype])
    over = (got - ref).abs() - (u * ref.abs() + tiny + PART[dtype] * mag)
    assert got.shape == ref.shape and torch.isfinite(got).all(), what
    assert not over.numel() or over.max() <= 0, (what, float(over.max()), int(over.argmax()))


def within32(got, ref, mag, dtype, what):
    """States: fp32 whatever the rows' type, products exact, pieces of 16 bits and more below 2^-20 of the largest."""
    got = cpu(got)
    assert got.shape == ref.shape and torch.isfinite(got).all(), what
    over = (got - ref).abs() - 2.0 ** -16 * mag - 2.0 ** -126
    assert over.max() <= 0, (what, float(over.max()))


def check_forward(q, k, v, g, offsets, at, S0, dtype, scale=0.3):
    o, last = B.spc_linear_attention_forward(q, k, v, g, offsets, scale=scale, initial_state=S0, want_state=True)
    ref, rlast = recur(cpu(q), cpu(k), cpu(v), cpu(g), at, scale, cpu(S0))
    mag, mlast = recur(cpu(q).abs(), cpu(k).abs(), cpu(v).abs(), cpu(g), at, scale, None if S0 is None else cpu(S0).abs())
    within(o, ref, mag, dtype, "out")
    within32(last, rlast, mlast, dtype, "state")
    return o, last


def reference_gradients(do, q, k, v, g, at, scale, S0, dS):
    """Gradients by differentiating the recurrence."""
    leaves = [t.detach().clone().requires_grad_() for t in (q, k, v, S0)]
    o, last = recur(leaves[0], leaves[1], leaves[2], g, at, scale, leaves[3])
    loss = (o * do).sum() + (last * dS).sum()
    return torch.autograd.grad(loss, leaves)


def check_backward(q, k, v, g, offsets, at, S0, dtype, scale=0.3, seed=9):
    gen = torch.Generator().manual_seed(seed)
    n, H, dv = q.shape[0], q.shape[1], v.shape[2]
    shape = (len(at) - 1, H, q.shape[2], dv)
    do = torch.randn(n, H, dv, generator=gen).to(dtype).cuda()
    dS = torch.randn(shape, generator=gen).cuda() if S0 is not None else None
    got = B.spc_linear_attention_backward(do, q, k, v, g, offsets, scale=scale, initial_state=S0, dstate=dS, want_dinitial=True)
    zero = torch.zeros(shape, dtype=torch.float64)
    c0, cS = (zero, zero) if S0 is None else (cpu(S0), cpu(dS))
    ref = reference_gradients(cpu(do), cpu(q), cpu(k), cpu(v), cpu(g), at, scale, c0, cS)
    mag = reference_gradients(cpu(do).abs(), cpu(q).abs(), cpu(k).abs(), cpu(v).abs(), cpu(g), at, scale, c0.abs(), cS.abs())
    for a, b, m, what in zip(got[:3], ref, mag, ("dq", "dk", "dv")):
        within(a, b, m, dtype, what)
    within32(got[3], ref[3], mag[3], dtype, "dinitial")
    return got


LENGTHS = [[1], [0, 1, 0], [2, 63, 64, 65], [31], [129, 0, 1, 300], [700]]
HEADS = [(1, 1, 64, 64), (4, 4, 16, 16), (2, 2, 32, 32), (4, 2, 24, 40), (6, 1, 64, 32), (2, 1, 5, 7), (1, 1, 128, 128), (2, 2, 1, 1), (3, 3, 33, 128), (2, 2, 128, 17)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("heads,kv,dk,dv", HEADS)
def test_forward(lengths, heads, kv, dk, dv, dtype):
    states = len(lengths) != 1 or lengths[0] == 31
    check_forward(*make(lengths, heads, kv, dk, dv, dtype, 7 * dk + dv, states), dtype)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("heads,kv,dk,dv", HEADS)
def test_backward(lengths, heads, kv, dk, dv, dtype):
    states = len(lengths) != 1 or lengths[0] == 31
    check_backward(*make(lengths, heads, kv, dk, dv, dtype, 7 * dk + dv + 1, states), dtype)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("layout", ["heads", "rows"])
def test_layouts(layout, dtype):
    """Heads outermost, and rows whose pitch is their width: the results are those of the column ranges, bit for bit."""
    a = make([200, 77], 4, 2, 32, 48, dtype, 3, True)
    b = make([200, 77], 4, 2, 32, 48, dtype, 3, True, layout=layout)
    fa, fb = (B.spc_linear_attention_forward(*t[:5], initial_state=t[6], want_state=True) for t in (a, b))
    assert all(torch.equal(p, q) for p, q in zip(fa, fb))
    do = torch.randn(277, 4, 48, device="cuda").to(dtype)
    far = torch.zeros(277, 4, 99, device="cuda", dtype=dtype)
    far[:, :, 3:51] = do
    ba = B.spc_linear_attention_backward(do, *a[:5], initial_state=a[6])
    out = tuple(torch.full((277, h, w + 1), 3.0, dtype=dtype, device="cuda")[:, :, 1:] for h, w in ((4, 32), (2, 32), (2, 48)))
    bb = B.spc_linear_attention_backward(far[:, :, 3:51], *b[:5], initial_state=b[6], out=out)
    assert all(torch.equal(p, q) for p, q in zip(ba[:3], bb[:3]))
    assert all((t._base[:, :, 0] == 3).all() for t in out)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("decay", [0.0, -1e-4, -3.0, -200.0, float("-inf")])
def test_decays(decay, dtype):
    a = make([150, 3], 2, 2, 32, 32, dtype, 5, True, decay=decay)
    check_forward(*a, dtype)
    q, k, v, g, offsets, at, S0 = a
    if decay > -1e9:
        check_backward(*a, dtype)
    else:  # every row by itself
        do = torch.randn(153, 2, 32, device="cuda").to(dtype)
        dS = torch.randn(S0.shape, device="cuda")
        dq, dk, dv, d0 = B.spc_linear_attention_backward(do, q, k, v, g, offsets, scale=0.3, initial_state=S0, dstate=dS, want_dinitial=True)
        within(dq, 0.3 * (cpu(do) * cpu(v)).sum(2, keepdim=True) * cpu(k), (cpu(do) * cpu(v)).abs().sum(2, keepdim=True) * cpu(k).abs(), dtype, "dq")
        assert (d0 == 0).all()


def test_several_chunks_a_segment():
    """Enough rows and heads for segments of more than 64 rows."""
    for heads, dtype in ((16, BF16), (12, F16)):
        a = make([9000, 1, 2501], heads, heads, 16, 16, dtype, 11, True)
        check_forward(*a, dtype)
    check_backward(*make([5000, 900], 16, 4, 16, 16, BF16, 12, True), BF16)


def test_scales_of_features():
    """Rows of tiny and of large features, and one channel far above the others: fp16's range is not that of sums and states."""
    for dtype in (F16, BF16):
        for kq, kv in ((1e-3, 1e-3), (30.0, 1e-2), (1e-2, 100.0)):
            q, k, v, g, offsets, at, _ = make([260], 2, 2, 32, 32, dtype, 21, False, decay=-0.01)
            q, k, v = (q.float() * kq).to(dtype), (k.float() * kq).to(dtype), (v.float() * kv).to(dtype)
            check_forward(q, k, v, g, offsets, at, None, dtype, scale=1.0)
        # values of one sign without a decay: states beyond fp16's largest number, outputs brought back by the scale
        q, k, v, g, offsets, at, _ = make([500], 1, 1, 16, 16, dtype, 22, False, decay=0.0)
        q, k, v = q.abs(), (q.abs() * 16).to(dtype), (v.abs() * 16).to(dtype)
        check_forward(q, k, v, g, offsets, at, None, dtype, scale=2.0 ** -12)


def test_gradients_against_differences():
    q, k, v, g, offsets, at, S0 = make([70, 20], 4, 2, 8, 12, F32, 31, True)
    gen = torch.Generator().manual_seed(1)
    do, dS = torch.randn(90, 4, 12, generator=gen).cuda(), torch.randn(2, 4, 8, 12, generator=gen).cuda()
    grads = B.spc_linear_attention_backward(do, q, k, v, g, offsets, scale=0.5, initial_state=S0, dstate=dS, want_dinitial=True)
    at64 = [cpu(t) for t in (q, k, v, S0)]

    def loss(x):
        o, last = recur(x[0], x[1], x[2], cpu(g), at, 0.5, x[3])
        return float((o * cpu(do)).sum() + (last * cpu(dS)).sum())

    for i, grad in enumerate(grads):
        d = torch.randn(at64[i].shape, generator=gen, dtype=torch.float64)
        hi, lo = list(at64), list(at64)
        hi[i], lo[i] = at64[i] + 1e-3 * d, at64[i] - 1e-3 * d
        num, ana = (loss(hi) - loss(lo)) / 2e-3, float((cpu(grad) * d).sum())  # (the loss is linear in each of the four)
        assert abs(num - ana) <= 2.0 ** -16 * float((cpu(grad) * d).abs().sum()) + 1e-9 * abs(loss(at64)), i


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("value", [float("inf"), float("nan"), float("-inf")])
def test_rows_that_are_not_finite_do_not_reach_earlier_ones(dtype, value):
    lengths, where = [200, 150], 137  # (in the middle of a chunk of the first scene)
    q, k, v, g, offsets, at, _ = make(lengths, 4, 2, 32, 32, dtype, 41, False, layout="rows")
    do = torch.randn(350, 4, 32, generator=torch.Generator().manual_seed(42)).to(dtype).cuda()
    o, last = B.spc_linear_attention_forward(q, k, v, g, offsets, scale=0.3, want_state=True)
    ref, _ = recur(cpu(q), cpu(k), cpu(v), cpu(g), at, 0.3)
    mag, _ = recur(cpu(q).abs(), cpu(k).abs(), cpu(v).abs(), cpu(g), at, 0.3)
    others = torch.cat([torch.arange(where), torch.arange(200, 350)])
    for t in (q, k, v):
        keep = t.clone()
        t[where, 0, 5] = value
        o2, last2 = B.spc_linear_attention_forward(q, k, v, g, offsets, scale=0.3, want_state=True)
        within(o2[others.cuda()], ref[others], mag[others], dtype, "earlier rows, other scenes")
        assert torch.equal(o2[:, 2:], o[:, 2:]) and torch.equal(last2[:, 2:], last[:, 2:]), "other heads"
        assert not torch.isfinite(o2[where, 0]).any() if t is not v else not torch.isfinite(o2[where, 0, 5])
        assert torch.equal(last2[1], last[1])
        t.copy_(keep)
    # backward: a gradient that is not finite reaches keys and values of rows up to its own only
    zero = torch.zeros(2, 4, 32, 32, dtype=torch.float64)
    refs = reference_gradients(cpu(do), cpu(q), cpu(k), cpu(v), cpu(g), at, 0.3, zero, zero)
    mags = reference_gradients(cpu(do).abs(), cpu(q).abs(), cpu(k).abs(), cpu(v).abs(), cpu(g), at, 0.3, zero, zero)
    do[where, 0, 3] = value
    got = B.spc_linear_attention_backward(do, q, k, v, g, offsets, scale=0.3)
    later = torch.arange(where + 1, 350)
    for i, rows in ((0, others), (1, later), (2, later)):
        within(got[i][rows.cuda()], refs[i][rows], mags[i][rows], dtype, ("dq", "dk", "dv")[i])


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("streams,heads,kv,dk,dv", [(1, 8, 8, 64, 64), (3, 4, 2, 24, 40), (17, 6, 1, 5, 7), (2, 2, 2, 128, 128), (5, 1, 1, 1, 1), (70, 2, 2, 33, 128), (9, 4, 4, 16, 16),
                                                    (4, 2, 2, 96, 32), (2, 3, 3, 128, 17)])
def test_step(streams, heads, kv, dk, dv, dtype):
    q, k, v, g, _, _, _ = make([streams], heads, kv, dk, dv, dtype, 51, False)
    S = torch.randn(streams, heads, dk, dv, device="cuda")
    before = cpu(S)
    at = list(range(streams + 1))
    o = B.spc_linear_attention_step(q, k, v, g, S, scale=0.3)
    ref, last = recur(cpu(q), cpu(k), cpu(v), cpu(g), at, 0.3, before)
    mag, mlast = recur(cpu(q).abs(), cpu(k).abs(), cpu(v).abs(), cpu(g), at, 0.3, before.abs())
    within(o, ref, mag, dtype, "out")
    within32(S, last, mlast, dtype, "state")


def test_steps_carry_a_scene_on():
    q, k, v, g, _, _, _ = make([300], 2, 2, 32, 32, F32, 61, False)
    whole, last = B.spc_linear_attention_forward(q, k, v, g, want_state=True)
    head, S = B.spc_linear_attention_forward(q[:290], k[:290], v[:290], g, want_state=True)
    rest = torch.cat([B.spc_linear_attention_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], g, S) for t in range(290, 300)])
    assert torch.allclose(torch.cat([head, rest]), whole, rtol=1e-4, atol=1e-4) and torch.allclose(S, last, rtol=1e-4, atol=1e-4)


def test_rows_in_no_scene_are_left_alone():
    q, k, v, g, _, _, _ = make([300], 2, 1, 16, 32, F16, 71, False)
    offsets = torch.tensor([20, 120, 250], dtype=torch.int32, device="cuda")
    clean = B.spc_linear_attention_forward(q[20:250], k[20:250], v[20:250], g, offsets - 20)[0]
    do = torch.randn(300, 2, 32, device="cuda").half()
    cg = B.spc_linear_attention_backward(do[20:250], q[20:250], k[20:250], v[20:250], g, offsets - 20)
    for t in (q, k, v, do):
        t[:20], t[250:] = float("nan"), float("nan")
    out = torch.full((300, 2, 32), 5.0, dtype=F16, device="cuda")
    B.spc_linear_attention_forward(q, k, v, g, offsets, out=out)
    assert (out[:20] == 5).all() and (out[250:] == 5).all()
    tol = 4 * U[F16] * clean.abs().max()  # (segments lie elsewhere, sums are associated otherwise)
    assert (out[20:250] - clean).abs().max() <= tol
    outs = tuple(torch.full(s, 5.0, dtype=F16, device="cuda") for s in ((300, 2, 16), (300, 1, 16), (300, 1, 32)))
    B.spc_linear_attention_backward(do, q, k, v, g, offsets, out=outs)
    assert (outs[0][:20] == 5).all() and (outs[0][250:] == 5).all()
    for a, b in zip(outs, cg):
        assert torch.isfinite(a[20:250]).all() and (a[20:250] - b).abs().max() <= 4 * U[F16] * b.abs().max()


@pytest.mark.parametrize("offsets", [[0, 1000, 300], [-5, 100, 300], [0, 200, 100, 300], [2 ** 31 - 1, -2 ** 31, 7], [300, 300, 300], [400, 500, 600]])
def test_offsets_that_are_none_stay_inside_the_rows(offsets):
    """Whatever offsets hold, nothing outside the tensors is touched: rows around them keep what they held, the states are written or left."""
    guard = torch.full((900, 2, 32), 5.0, dtype=F16, device="cuda")
    q, k, v, g, _, _, _ = make([300], 2, 2, 32, 32, F16, 81, False)
    at = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    B.spc_linear_attention_forward(q, k, v, g, at, out=guard[300:600], want_state=True)
    outs = tuple(torch.full((900, 2, 32), 5.0, dtype=F16, device="cuda") for _ in range(3))
    B.spc_linear_attention_backward(v, q, k, v, g, at, out=tuple(t[300:600] for t in outs), want_dinitial=True)
    for t in (guard, *outs):
        assert (t[:300] == 5).all() and (t[600:] == 5).all()


def test_many_scenes():
    """More scenes times heads than a grid has rows, three rows each, the last longer than a segment."""
    b, H, d = 20_000, 4, 16
    lengths = [3] * b + [300]
    q, k, v, g, offsets, _, S0 = make(lengths, H, H, d, d, F32, 85, True)
    o, last = B.spc_linear_attention_forward(q, k, v, g, offsets, scale=0.3, initial_state=S0, want_state=True)
    l, S = torch.exp(cpu(g))[:, None, None], cpu(S0[:b])
    qs, ks, vs = (cpu(t[:3 * b]).reshape(b, 3, H, d) for t in (q, k, v))
    for t in range(3):
        S = l * S + ks[:, t, :, :, None] * vs[:, t, :, None, :]
        ref = 0.3 * (qs[:, t, :, :, None] * S).sum(2)
        assert (cpu(o[t:3 * b:3]) - ref).abs().max() <= 2.0 ** -16 * 16 * 64  # (sixteen products of values below 4 and states below 16)
    assert (cpu(last[:b]) - S).abs().max() <= 2.0 ** -16 * 64
    whole, end = recur(cpu(q[3 * b:]), cpu(k[3 * b:]), cpu(v[3 * b:]), cpu(g), [0, 300], 0.3, cpu(S0[b:]))
    mag, emag = recur(cpu(q[3 * b:]).abs(), cpu(k[3 * b:]).abs(), cpu(v[3 * b:]).abs(), cpu(g), [0, 300], 0.3, cpu(S0[b:]).abs())
    within(o[3 * b:], whole, mag, F32, "the long scene")
    within32(last[b:], end, emag, F32, "its state")


def test_no_rows_and_empty_scenes():
    q, k, v, g, _, _, _ = make([0], 2, 2, 16, 16, F32, 91, False)
    S0, dS = torch.randn(3, 2, 16, 16, device="cuda"), torch.randn(3, 2, 16, 16, device="cuda")
    none = torch.zeros(4, dtype=torch.int32, device="cuda")
    o, last = B.spc_linear_attention_forward(q, k, v, g, none, initial_state=S0, want_state=True)
    assert o.shape == (0, 2, 16) and torch.equal(last, S0)
    assert (B.spc_linear_attention_forward(q, k, v, g, none, want_state=True)[1] == 0).all()
    dq, dk, dv, d0 = B.spc_linear_attention_backward(o, q, k, v, g, none, initial_state=S0, dstate=dS, want_dinitial=True)
    assert torch.equal(d0, dS) and dq.numel() == dk.numel() == dv.numel() == 0
    assert B.spc_linear_attention_step(q, k, v, g, S0[:0]).shape == (0, 2, 16)


def test_same_bits_every_time_and_on_another_stream():
    q, k, v, g, offsets, _, S0 = make([5000, 800], 8, 2, 32, 32, BF16, 101, True)
    do = torch.randn(5800, 8, 32, device="cuda").to(BF16)

    def step():
        return *B.spc_linear_attention_forward(q, k, v, g, offsets, initial_state=S0, want_state=True), \
            *B.spc_linear_attention_backward(do, q, k, v, g, offsets, initial_state=S0, want_dinitial=True)

    first = step()
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(other):
            again = step()
        other.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_recorded():
    q, k, v, g, offsets, _, _ = make([900, 300], 4, 2, 32, 32, F16, 111, False, layout="rows")
    do = torch.randn(1200, 4, 32, device="cuda").half()

    def step():
        return B.spc_linear_attention_forward(q, k, v, g, offsets)[0], *B.spc_linear_attention_backward(do, q, k, v, g, offsets)[:3]

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = step()
    for r in range(3):
        q.normal_()
        offsets.copy_(torch.tensor([0, 500 + 100 * r, 1200], dtype=torch.int32))  # (scenes of other lengths, the same record)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_rows_far_apart():
    """Row offsets beyond 32 bits, in and out."""
    n, pitch = 300, 16_000_000
    wide = torch.empty(n * pitch, dtype=BF16, device="cuda")
    q, k, v = (wide.as_strided((n, 2, 32), (pitch, 32, 1), 64 * i) for i in range(3))
    for t in (q, k, v):
        t.copy_(torch.randn(n, 2, 32))
    g = torch.tensor([-0.1, -0.01], device="cuda")
    near = [t.contiguous() for t in (q, k, v)]
    far = wide.as_strided((n, 2, 32), (pitch, 32, 1), 64 * 3)
    B.spc_linear_attention_forward(q, k, v, g, out=far)
    want = B.spc_linear_attention_forward(*near, g)[0]
    assert torch.equal(far, want)
    a, b = B.spc_linear_attention_backward(far, q, k, v, g), B.spc_linear_attention_backward(want, *near, g)
    assert all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))


def test_broadcast_inputs():
    q, k, v, g, offsets, at, _ = make([130], 4, 4, 16, 16, BF16, 121, False, layout="rows")
    one = k[:, :1].expand(130, 4, 16)  # (a pitch of zero between heads)
    same = one.contiguous()
    assert torch.equal(B.spc_linear_attention_forward(q, one, v, g, offsets)[0], B.spc_linear_attention_forward(q, same, v, g, offsets)[0])
    a, b = (B.spc_linear_attention_backward(v, q, t, v, g, offsets) for t in (one, same))
    assert all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))


@pytest.mark.parametrize("key_bits", [32, 64])
def test_batch_offsets(key_bits):
    gen = torch.Generator().manual_seed(2)
    counts = [300, 0, 1, 5000, 0, 77]
    rows = torch.cat([torch.cat([torch.full((c, 1), b), torch.randint(0, 60, (c, 3), generator=gen)], 1) for b, c in enumerate(counts)]).to(torch.int32)
    rows = rows[torch.randperm(len(rows), generator=gen)].cuda()
    desc = B.spc_pack_desc_fit([0, 0, 0], [59, 59, 59], 6, 1, 1, key_bits)
    keys, _ = B.spc_pack_coords(rows, desc)
    assert B.spc_batch_offsets(keys, desc, 6).tolist() == [0] + list(itertools.accumulate(counts))
    assert B.spc_batch_offsets(keys, desc, 2).tolist() == [0, 300, 300]
    one = B.spc_pack_desc_fit([0, 0, 0], [59, 59, 59], 1, 1, 1, key_bits)
    keys, _ = B.spc_pack_coords(rows * torch.tensor([0, 1, 1, 1], dtype=torch.int32, device="cuda"), one)
    assert B.spc_batch_offsets(keys, one, 1).tolist() == [0, sum(counts)]
    assert B.spc_batch_offsets(keys[:0], one, 1).tolist() == [0, 0]


def test_refusals():
    q, k, v, g, offsets, _, S0 = make([40], 4, 2, 16, 16, F16, 131, True)

    def refused(code, **change):
        a = dict(q=q, k=k, v=v, log_decay=g, offsets=offsets)
        a.update(change)
        with pytest.raises(B.SpcError) as e:
            B.spc_linear_attention_forward(**a)
        assert e.value.code == code

    refused(B.ERR_UNSUPPORTED, q=torch.zeros(40, 4, 129, device="cuda").half(), k=torch.zeros(40, 2, 129, device="cuda").half())
    refused(B.ERR_UNSUPPORTED, v=torch.zeros(40, 2, 129, device="cuda").half())
    refused(B.ERR_ARG, k=torch.zeros(40, 3, 16, device="cuda").half(), v=torch.zeros(40, 3, 16, device="cuda").half())  # 4 heads over 3
    refused(B.ERR_ARG, scale=float("nan"))
    refused(B.ERR_ARG, out=torch.zeros(40, 1, 16, device="cuda").half().expand(40, 4, 16))  # heads on top of each other
    refused(B.ERR_ARG, out=torch.zeros(1, 4, 16, device="cuda").half().expand(40, 4, 16))
    for change in (dict(q=q.float()), dict(k=k[:39]), dict(log_decay=g[:3]), dict(log_decay=g.double()), dict(offsets=offsets.long()),
                   dict(initial_state=S0[:, :3]), dict(initial_state=S0.half()), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2))):
        a = dict(q=q, k=k, v=v, log_decay=g, offsets=offsets)
        a.update(change)
        with pytest.raises(AssertionError):
            B.spc_linear_attention_forward(**a)
    L, p, s = B.lib(), q.data_ptr(), S0.data_ptr()
    d, r = B.AttnDesc(0, 1, 40, 4, 2, 16, 16, 0.25), B.AttnRows(p, 128, 16)
    call = lambda d=d, q=r, k=r, v=r, g=g.data_ptr(), at=None, o=r: L.spc_linear_attention_forward(d, q, k, v, g, at, None, o, None, None)
    assert call(g=None) == B.ERR_ARG and call(d=None) == B.ERR_ARG and call(q=None) == B.ERR_ARG and call(o=B.AttnRows(None, 128, 16)) == B.ERR_ARG
    assert call(q=B.AttnRows(p + 1, 128, 16)) == B.ERR_ARG and call(k=B.AttnRows(p, -1, 16)) == B.ERR_ARG
    for bad in ((3, 1, 40, 4, 2, 16, 16), (0, 0, 40, 4, 2, 16, 16), (0, 2, 40, 4, 2, 16, 16), (0, 1, -1, 4, 2, 16, 16), (0, 1, 40, 0, 1, 16, 16), (0, 1, 40, 4, 0, 16, 16),
                (0, 1, 40, 4, 2, 0, 16)):
        assert call(d=B.AttnDesc(*bad, 0.25)) == B.ERR_ARG, bad
    assert call(d=B.AttnDesc(0, 1, 1 << 31, 4, 2, 16, 16, 0.25)) == B.ERR_UNSUPPORTED
    assert call(d=B.AttnDesc(0, 50_001, 40, 4, 2, 16, 16, 0.25), at=offsets.data_ptr()) == B.ERR_UNSUPPORTED  # scenes times heads
    assert L.spc_linear_attention_step(B.AttnDesc(0, 1, 1 << 23, 4, 2, 16, 16, 0.25), r, r, r, g.data_ptr(), s, r, None) == B.ERR_UNSUPPORTED
    assert L.spc_linear_attention_step(d, r, r, r, g.data_ptr(), None, r, None) == B.ERR_ARG
    assert L.spc_linear_attention_backward(d, r, r, r, r, g.data_ptr(), None, None, None, r, r, None, None, None) == B.ERR_ARG
    assert L.spc_batch_offsets(s, 5, None, 1, s, None) == B.ERR_ARG


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("decay", [0.0, -1 / 4096, -1 / 256])
def test_long_memories_keep_their_bits(dtype, decay):
    """A state of up to some 300 chunks (2-norms over a head).  A chunk's sum: up to 64 roundings of 2^-24 of sums that grow as a random walk, together some 3 of 2^-24.  Adding up the
    chunks, 2 roundings each of a sum that grows likewise: some sqrt(300) / sqrt(3) / 2 = 5.  Together below 8, 2^-21; a decay whose rounding met all of them would add up to 64 halves, and
    roundings at every product of a memory of 4096 rows and more some 12."""
    n, heads, d = 20_000, 64, 16
    gen = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(n, heads, d, generator=gen).to(dtype) for _ in range(3))
    g = torch.full((heads,), decay)
    _, last = B.spc_linear_attention_forward(q.cuda(), k.cuda(), v.cuda(), g.cuda(), want_state=True)
    w = torch.exp(g[0].double() * torch.arange(n - 1, -1, -1))[:, None]
    for h in range(heads):
        ref = (k[:, h].double() * w).T @ v[:, h].double()
        assert (cpu(last[0, h]) - ref).norm() <= 2.0 ** -21 * ref.norm(), h


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("heads,kv", [(2, 2), (2, 1), (6, 2)])
@pytest.mark.parametrize("at", [[20, 120, 250], [0, 0, 299], [300, 300], [0, 0], [7, 7, 8]], ids=str)
def test_gradients_of_rows_in_no_scene_are_left_alone(at, heads, kv, dtype):
    """All three gradients, with heads of their own and with shared ones, whose parts per head lie in scratch that other calls have used.  Rows of scenes are held against
    the recurrence."""
    q, k, v, g, _, _, _ = make([300], heads, kv, 16, 24, dtype, 141, False, layout="rows")
    do = torch.randn(300, heads, 24, generator=torch.Generator().manual_seed(142)).to(dtype).cuda()
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    for _ in range(2):  # (scratch full of NaN, if the next call takes its block)
        B.spc_linear_attention_backward(do * float("nan"), q, k, v, g)
    lo, hi = at[0], at[-1]
    inside = [cpu(t)[lo:hi] for t in (do, q, k, v)]
    for t in (do, q, k, v):
        t[:lo], t[hi:] = float("nan"), float("nan")
    outs = tuple(torch.full((300, h, w), 5.0, dtype=dtype, device="cuda") for h, w in ((heads, 16), (kv, 16), (kv, 24)))
    B.spc_linear_attention_backward(do, q, k, v, g, offsets, scale=0.3, out=outs)
    for t, what in zip(outs, ("dq", "dk", "dv")):
        assert (t[:lo] == 5).all() and (t[hi:] == 5).all(), what
    if hi == lo:
        return
    zero = torch.zeros(len(at) - 1, heads, 16, 24, dtype=torch.float64)
    rel = [a - lo for a in at]
    refs = reference_gradients(inside[0], *inside[1:], cpu(g), rel, 0.3, zero, zero)
    mags = reference_gradients(*[t.abs() for t in inside], cpu(g), rel, 0.3, zero, zero)
    for t, ref, mag, what in zip(outs, refs, mags, ("dq", "dk", "dv")):
        within(t[lo:hi], ref, mag, dtype, what)


@pytest.mark.parametrize("backward", [False, True])
def test_scenes_of_nearly_all_the_rows_there_can_be(backward):
    """2^31 - 1 rows of one scene: its rows and one segment's more pass 31 bits.  One row for all inputs; a decay of a half, so the sums are at 2 from row 24 on."""
    n = (1 << 31) - 1
    one = torch.ones(1, 1, 1, dtype=F16, device="cuda").expand(n, 1, 1)
    g = torch.full((1,), 0.5, device="cuda").log()
    if backward:
        outs = tuple(torch.full((n, 1, 1), 5.0, dtype=F16, device="cuda") for _ in range(3))
        dstate = torch.zeros(1, 1, 1, 1, device="cuda")
        first = B.spc_linear_attention_backward(one, one, one, one, g, scale=1.0, dstate=dstate, want_dinitial=True, out=outs)[3]
        assert abs(float(first) - 1) < 1e-6
        checks = [(outs[0], False), (outs[1], True), (outs[2], True)]
    else:
        out, last = B.spc_linear_attention_forward(one, one, one, g, scale=1.0, want_state=True)
        assert abs(float(last) - 2) < 1e-6
        checks = [(out, False)]
    for t, reverse in checks:
        t = t.view(-1)
        ends = t[-64:].flip(0) if reverse else t[:64]
        want = 2 - torch.exp2(-torch.arange(64.0)).cuda()
        assert (ends.float() - want).abs().max() <= 2 * U[F16] * 2
        inner = t[:-64] if reverse else t[64:]
        assert inner.min() == 2 and inner.max() == 2


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("small,large", [(0.1, 100.0), (0.01, 1000.0)])
@pytest.mark.parametrize("decay", [-1.0, -0.25, -1 / 256])
@pytest.mark.parametrize("which", ["qkv", "k", "v", "kv"])
def test_rows_of_unlike_scales(which, decay, small, large, dtype):
    """Every sixteenth row far above the others, so that far rows count as much as near ones: each product is held against the sum of the magnitudes that it is made of."""
    q, k, v, g, offsets, at, S0 = make([150, 70], 2, 1, 16, 24, dtype, 151, True, decay=decay)
    by = torch.where(torch.arange(220) % 16 == 3, large, small).cuda()[:, None, None]
    q, k, v = (t.float() * (by if name in which else 1.0) for name, t in zip("qkv", (q, k, v)))
    scale = 30 / large ** len(which) if dtype == F16 else 0.3  # (outputs of fp16 below its largest number)
    check_forward(q.to(dtype), k.to(dtype), v.to(dtype), g, offsets, at, S0, dtype, scale=scale)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_gradients_of_rows_of_unlike_scales(dtype):
    q, k, v, g, offsets, at, S0 = make([150, 70], 4, 2, 16, 24, dtype, 152, True, decay=-0.5)
    by = torch.where(torch.arange(220) % 16 == 3, 10.0, 0.02).cuda()[:, None, None]
    check_backward(*((t.float() * by).to(dtype) for t in (q, k, v)), g, offsets, at, S0, dtype)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_channels_of_unlike_scales(dtype):
    """One channel of the keys far above the others, which queries read as far below them."""
    q, k, v, g, offsets, at, _ = make([200], 2, 2, 32, 32, dtype, 153, False, decay=-0.02)
    by = torch.where(torch.arange(32) == 5, 1000.0, 0.01).cuda()
    check_forward((q.float() / by / 10).to(dtype), (k.float() * by).to(dtype), v, g, offsets, at, None, dtype, scale=1.0)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("decay", [-1.0, -0.4])
@pytest.mark.parametrize("rows", [64, 50])
def test_values_before_rows_of_zeros(rows, decay, dtype):
    """Values of a chunk's first rows and zeros behind them: the state is what the decay has left of the former."""
    q, k, v, g, offsets, at, _ = make([rows], 2, 2, 16, 32, dtype, 154, False, decay=decay, layout="rows")
    v[16:] = 0
    check_forward(q, k, v, g, offsets, at, None, dtype)
    do = torch.randn(rows, 2, 32, generator=torch.Generator().manual_seed(155)).to(dtype).cuda()
    do[:-16] = 0  # (backward in time)
    first = B.spc_linear_attention_backward(do, q, k, v, g, offsets, scale=0.3, want_dinitial=True)[3]
    zero = torch.zeros(1, 2, 16, 32, dtype=torch.float64)
    ref = reference_gradients(cpu(do), cpu(q), cpu(k), cpu(v), cpu(g), at, 0.3, zero, zero)[3]
    mag = reference_gradients(cpu(do).abs(), cpu(q).abs(), cpu(k).abs(), cpu(v).abs(), cpu(g), at, 0.3, zero, zero)[3]
    within32(first, ref, mag, dtype, "dinitial")


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("decay", [-1 / 4096, -1 / 3000, -1 / 256, -0.3])
def test_long_streams_keep_their_bits(dtype, decay):
    """20 000 steps of one stream (2-norms over a head).  A step rounds its state once, by up to half of 2^-23 of it, 2^-23 / sqrt(12) on average, and a memory of M = 1 / -decay
    rows adds up M / 2 squares of that: sqrt(M / 2) 2^-24.8, twice that allowed.  (Short memories: no less than a step's own roundings, of its product and its decay.)  One
    rounding of the decay would add up to M / 2 of 2^-24, 45 times as much at M = 4096.  And the scene call over the same rows, which has its own 2^-21."""
    n, heads, d = 20_000, 4, 16
    gen = torch.Generator().manual_seed(6)
    q, k, v = (torch.randn(n, heads, d, generator=gen).to(dtype) for _ in range(3))
    g = torch.full((heads,), decay)
    S = torch.zeros(1, heads, d, d, device="cuda")
    qg, kg, vg, gg, out = q.cuda(), k.cuda(), v.cuda(), g.cuda(), torch.empty(1, heads, d, dtype=dtype, device="cuda")
    for t in range(n):
        B.spc_linear_attention_step(qg[t:t + 1], kg[t:t + 1], vg[t:t + 1], gg, S, out=out)
    _, last = B.spc_linear_attention_forward(qg, kg, vg, gg, want_state=True)
    w = torch.exp(g[0].double() * torch.arange(n - 1, -1, -1))[:, None]
    bound = 2 * max(0.5 / -decay, 4.0) ** 0.5 * 2.0 ** -24.8
    for h in range(heads):
        ref = (k[:, h].double() * w).T @ v[:, h].double()
        assert (cpu(S[0, h]) - ref).norm() <= bound * ref.norm(), h
        assert (cpu(S[0, h]) - cpu(last[0, h])).norm() <= (bound + 2.0 ** -21) * ref.norm(), h


def without_states(lengths, heads, kv, dk, dv, dtype, seed, decay=None, initial=False):
    """The calls that return no state (bf16 keeps fewer bits of the states in between then), outputs and gradients within the same bounds."""
    q, k, v, g, offsets, at, S0 = make(lengths, heads, kv, dk, dv, dtype, seed, initial, decay=decay)
    do = torch.randn(q.shape[0], heads, dv, generator=torch.Generator().manual_seed(seed + 1)).to(dtype).cuda()
    zero = torch.zeros(len(at) - 1, heads, dk, dv, dtype=torch.float64)
    first = zero if S0 is None else cpu(S0)
    o, last = B.spc_linear_attention_forward(q, k, v, g, offsets, scale=0.3, initial_state=S0)
    assert last is None
    within(o, recur(cpu(q), cpu(k), cpu(v), cpu(g), at, 0.3, first)[0], recur(cpu(q).abs(), cpu(k).abs(), cpu(v).abs(), cpu(g), at, 0.3, first.abs())[0], dtype, "out")
    got = B.spc_linear_attention_backward(do, q, k, v, g, offsets, scale=0.3, initial_state=S0)
    assert got[3] is None
    refs = reference_gradients(cpu(do), cpu(q), cpu(k), cpu(v), cpu(g), at, 0.3, first, zero)
    mags = reference_gradients(cpu(do).abs(), cpu(q).abs(), cpu(k).abs(), cpu(v).abs(), cpu(g), at, 0.3, first.abs(), zero)
    for a, b, m, what in zip(got[:3], refs, mags, ("dq", "dk", "dv")):
        within(a, b, m, dtype, what)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("lengths", [[2, 63, 64, 65], [129, 0, 1, 300], [700]], ids=str)
@pytest.mark.parametrize("heads,kv,dk,dv", HEADS)
def test_without_states(lengths, heads, kv, dk, dv, dtype):
    without_states(lengths, heads, kv, dk, dv, dtype, 7 * dk + dv + 2)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("decay", [0.0, -1e-4, -0.05, -3.0, -200.0])
def test_decays_without_states(decay, dtype):
    without_states([150, 3, 400], 2, 2, 32, 32, dtype, 161, decay=decay, initial=True)


def test_several_chunks_a_segment_without_states():
    without_states([5000, 900], 16, 4, 16, 16, BF16, 162)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("decay", [0.0, -1 / 4096])
def test_outputs_of_long_memories_without_states(dtype, decay):
    """The last rows of one head of 20 000 (as in the test of their states; here what nobody keeps the state of)."""
    n, heads, d = 20_000, 8, 32
    gen = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn(n, heads, d, generator=gen).to(dtype) for _ in range(3))
    g = torch.full((heads,), decay)
    o, _ = B.spc_linear_attention_forward(q.cuda(), k.cuda(), v.cuda(), g.cuda(), scale=0.01)
    for t in (n - 1, n - 70, 12_345):
        w = torch.exp(g[0].double() * torch.arange(t, -1, -1))[:, None]
        for h in range(0, heads, 3):
            a, b, c = q[t, h].double(), k[:t + 1, h].double(), v[:t + 1, h].double()
            within(o[t, h], 0.01 * ((b @ a)[:, None] * w * c).sum(0), 0.01 * ((b.abs() @ a.abs())[:, None] * w * c.abs()).sum(0), dtype, (t, h))


@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_many_scenes_each_within_its_bounds(dtype, states):
    """Scenes of three rows (and an empty one, and a long one), each held against the recurrence with the bounds of all other results."""
    b, H, d = 3000, 4, 16
    lengths = [3] * b + [0, 300]
    q, k, v, g, offsets, _, S0 = make(lengths, H, 2, d, d, dtype, 163, True)
    o, last = B.spc_linear_attention_forward(q, k, v, g, offsets, scale=0.3, initial_state=S0, want_state=states)
    l = torch.exp(cpu(g))[:, None, None]
    qs, ks, vs = (cpu(t[:3 * b]).reshape(b, 3, -1, d) for t in (q, k, v))
    ks, vs = ks.repeat_interleave(2, 2), vs.repeat_interleave(2, 2)
    S, M = cpu(S0[:b]), cpu(S0[:b]).abs()
    for t in range(3):
        S, M = l * S + ks[:, t, :, :, None] * vs[:, t, :, None, :], l * M + (ks[:, t, :, :, None] * vs[:, t, :, None, :]).abs()
        ref, mag = (0.3 * (x[:, t, :, :, None] * y).sum(2) for x, y in ((qs, S), (qs.abs(), M)))
        within(o[t:3 * b:3], ref, mag, dtype, t)
    if states:
        within32(last[:b], S, M, dtype, "states")
        assert torch.equal(last[b], S0[b])
