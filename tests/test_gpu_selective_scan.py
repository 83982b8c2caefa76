"""Selective scan along scenes, forward, backward and by single rows, against the recurrence in 64 bits, a row at a time.

Tolerances are carried along: every quantity is a pair of its magnitude (the same sums over magnitudes) and its error.  A product's error is |f| eg + |g| ef, and each step
adds R = 2^-20 of the magnitude: up to 16 roundings of 2^-24 (sums over states or channels of a workgroup are trees or chains of as many at most, step sizes a series of some ten
operations).  A decay exp(d A) has its exponent's error, 2^-20 (1 + |d A|) of itself, so that a memory of M rows collects M of those.  Columns are added up in chains
of at most 200 rows and parts: 2^-16.  The last rounding is half a unit in the last place of the rows' type."""
import pytest
import torch

from paper_2511_20834_amd import binding as B

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
U = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}
# Spacing of fp16 near zero; a term below 2^-126 is zero in 32 bits (states of exp(-140) are met below), and a result adds up at most 2^10 of them times factors up to 2^6.
TINY = {F16: 2.0 ** -24, BF16: 2.0 ** -110, F32: 2.0 ** -110}
R, COLUMN = 2.0 ** -20, 2.0 ** -16


class Mag:
    """Value, magnitude and error of a tensor."""

    def __init__(self, v, m=None, e=None):
        self.v, self.m, self.e = v, v.abs() if m is None else m, torch.zeros_like(v) if e is None else e

    def __mul__(self, o):
        m = self.m * o.m
        return Mag(self.v * o.v, m, self.m * o.e + self.e * o.m + R * m)

    def __add__(self, o):
        m = self.m + o.m
        return Mag(self.v + o.v, m, self.e + o.e + R * m)

    def sum(self, dim, extra=R):
        return Mag(self.v.sum(dim), self.m.sum(dim), self.e.sum(dim) + extra * self.m.sum(dim))

    def __getitem__(self, i):
        return Mag(self.v[i], self.m[i], self.e[i])

    def map(self, f):
        return Mag(f(self.v), f(self.m), f(self.e))


def stack(rows):
    return Mag(*(torch.stack([getattr(r, k) for r in rows]) for k in ("v", "m", "e")))


def silu_and_slope(z):
    p = torch.sigmoid(z)
    s, d = z * p, p * (1 + z * (1 - p))
    return Mag(s, e=s.abs() * (z.abs() + 8) * 2.0 ** -22), Mag(d, e=(1 + z.abs()) * (z.abs() + 8) * 2.0 ** -21)


def reference(u, dt, A, Bm, Cm, skip, gate, bias, at, softplus, initial, dout=None, dlast=None):
    """All results as Mag, on the host."""
    up = lambda t: None if t is None else t.double().cpu()  # noqa: E731
    u, dt, A, Bm, Cm, skip, gate, bias, initial, dout, dlast = map(up, (u, dt, A, Bm, Cm, skip, gate, bias, initial, dout, dlast))
    n, c = u.shape
    G, N = Bm.shape[1:]
    spread = lambda t: t.repeat_interleave(c // G, 1)  # noqa: E731
    raw = dt + (0 if bias is None else bias)
    er = R * (dt.abs() + (0 if bias is None else bias.abs()))
    if softplus:
        d = torch.logaddexp(raw, torch.zeros_like(raw))
        delta = Mag(d, e=torch.sigmoid(raw) * er + R * (1 + raw.abs()) * d)
        slope = Mag(torch.sigmoid(raw), e=R * (1 + raw.abs()) + er)
    else:
        delta, slope = Mag(raw, e=er), Mag(torch.ones_like(raw))
    w = delta.v[..., None] * A
    a = Mag(torch.exp(w), e=torch.exp(w) * (R * (1 + w.abs()) + delta.e[..., None] * A.abs()))
    x = delta * Mag(u)
    Bf, Cf = spread(Bm), spread(Cm)
    bx = Mag(x.v[..., None], x.m[..., None], x.e[..., None]) * Mag(Bf)
    scenes = list(zip(at, at[1:]))
    zero = Mag(torch.zeros(c, N, dtype=torch.float64))
    h, before, last = [None] * n, [None] * n, []
    for b, (lo, hi) in enumerate(scenes):
        s = zero if initial is None else Mag(initial[b])
        for t in range(lo, hi):
            before[t] = s
            s = a[t] * s + bx[t]
            h[t] = s
        last.append(s)
    out = {"state": stack(last)}
    if not n:
        return out
    H = stack(h)
    y = (H * Mag(Cf)).sum(2)
    if skip is not None:
        y = y + Mag(skip) * Mag(u)
    act, act_slope = silu_and_slope(gate) if gate is not None else (None, None)
    out["y"] = y if gate is None else y * act
    if dout is None:
        return out
    dout = Mag(dout)
    dy = dout
    if gate is not None:
        out["gate"] = dout * y * act_slope
        dy = dout * act
    col = lambda t: Mag(t.v[..., None], t.m[..., None], t.e[..., None])  # noqa: E731
    direct = col(dy) * Mag(Cf)
    q, first = [None] * n, []
    for b, (lo, hi) in enumerate(scenes):
        r = zero if dlast is None else Mag(dlast[b])
        for t in range(hi - 1, lo - 1, -1):
            q[t] = direct[t] + r
            r = a[t] * q[t]
        first.append(r)
    out["initial"] = stack(first)
    Q, P = stack(q), stack(before)
    groups = lambda t: t.map(lambda v: v.unflatten(1, (G, c // G))).sum(2)  # noqa: E731
    out["C"], out["B"] = groups(H * col(dy)), groups(Q * col(x))
    p = Q * a * P
    dx = (Q * Mag(Bf)).sum(2)
    ddt = (Mag(u) * dx + (p * Mag(A.expand_as(p.v))).sum(2)) * slope
    out["dt"], out["dt_bias"] = ddt, ddt.sum(0, COLUMN)
    out["u"] = delta * dx if skip is None else delta * dx + Mag(skip) * dy
    out["A"] = (p * col(delta)).sum(0, COLUMN)
    out["skip"] = (dy * Mag(u)).sum(0, COLUMN)
    return out


def close(got, ref, dtype, what):
    got = got.double().cpu()
    assert got.shape == ref.v.shape, (what, got.shape, ref.v.shape)
    if not got.numel():
        return
    over = (got - ref.v).abs() - (ref.e + U[dtype] * ref.v.abs() + TINY[dtype])
    assert torch.isfinite(got).all() and over.max() <= 0, (what, float(over.max()), int(over.argmax()))


def matrix(n, c, dtype, gen, pitch=0, first=0, scale=1.0):
    t = (scale * torch.randn(n, c, generator=gen)).to(dtype).cuda()
    if not pitch:
        return t
    wide = torch.full((n, c + pitch), float("nan"), dtype=dtype, device="cuda")
    wide[:, first:first + c] = t
    return wide[:, first:first + c]


def case(lengths, c, G, N, dtype, gate=True, states=True, skip=True, bias=True, pitch=0, first=0, seed=1):
    gen = torch.Generator().manual_seed(seed + 7 * c + N)
    n, b = sum(lengths), len(lengths)
    r = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
    step = torch.exp(torch.rand(c, generator=gen) * 4.6 - 6.9).cuda()  # 1e-3 to 0.1
    low = matrix(n, 5 + 2 * G * N, dtype, gen)
    k = {"u": matrix(n, c, dtype, gen, pitch, first), "dt": matrix(n, c, dtype, gen, pitch, first, 0.5), "A": -torch.exp(r(c, N)) * (1 + torch.arange(N).cuda()),
         "B": low[:, 5:5 + G * N].unflatten(1, (G, N)), "C": low[:, 5 + G * N:].unflatten(1, (G, N)), "skip": r(c) if skip else None,
         "gate": matrix(n, c, dtype, gen, pitch, first) if gate else None, "dt_bias": (step + torch.log(-torch.expm1(-step))) if bias else None,
         "offsets": torch.tensor([0, *lengths]).cumsum(0).to(torch.int32).cuda(), "initial_state": r(b, c, N) if states else None}
    return k, matrix(n, c, dtype, gen, pitch, first), r(b, c, N) if states else None


def wanted(k, softplus=True, dout=None, dstate=None):
    return reference(k["u"], k["dt"], k["A"], k["B"], k["C"], k["skip"], k["gate"], k["dt_bias"], k["offsets"].tolist(), softplus, k["initial_state"], dout, dstate)


def check_all(k, dout, dstate, softplus=True):
    dtype = k["u"].dtype
    ref = wanted(k, softplus, dout, dstate)
    y, state = B.spc_selective_scan_forward(**k, softplus=softplus, want_state=True)
    close(state, ref["state"], F32, "state")
    if k["u"].shape[0]:
        close(y, ref["y"], dtype, "y")
    g = B.spc_selective_scan_backward(dout, **k, softplus=softplus, dstate=dstate, want_dinitial=True)
    for name in g._fields:
        if name == "initial" or (k["u"].shape[0] and getattr(g, name) is not None):
            close(getattr(g, name), ref[name], F32 if name in ("A", "skip", "dt_bias", "initial") else dtype, name)
    assert (g.gate is None) == (k["gate"] is None) and (g.skip is None) == (k["skip"] is None) and (g.dt_bias is None) == (k["dt_bias"] is None)
    again = B.spc_selective_scan_backward(dout, **k, softplus=softplus, dstate=dstate)
    assert again.initial is None and all(torch.equal(p, q) for p, q in zip(g[:-1], again[:-1]) if p is not None)
    assert torch.equal(B.spc_selective_scan_forward(**k, softplus=softplus)[0], y)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("lengths", [[1], [2], [17], [300], [0, 5, 1, 0, 130, 3]], ids=str)
@pytest.mark.parametrize("c,G,N", [(64, 1, 16), (1, 1, 1), (130, 2, 8), (65, 1, 3), (90, 3, 17), (200, 1, 4), (20, 1, 64), (256, 1, 16)])
def test_forward_and_backward(lengths, c, G, N, dtype):
    check_all(*case(lengths, c, G, N, dtype))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("gate,states,skip,bias,pitch,first", [(False, False, False, False, 0, 0), (True, False, True, False, 7, 3), (False, True, False, True, 1, 1), (True, True, False, True, 0, 0)])
@pytest.mark.parametrize("N", [16, 32])
def test_what_may_be_missing(gate, states, skip, bias, pitch, first, softplus, N, dtype):
    k, dout, dstate = case([100, 70], 70, 1, N, dtype, gate, states, skip, bias, pitch, first)
    if not softplus:  # (step sizes are what the caller says: above zero here)
        k["dt"] = (0.05 * k["dt"].abs()).to(dtype)
        k["dt_bias"] = None if k["dt_bias"] is None else 0.01 * k["dt_bias"].abs()
    check_all(k, dout, dstate, softplus)


@pytest.mark.parametrize("N", [8, 16, 33])
def test_many_segments(N):
    """Segments of every scene are chained; channels of two blocks."""
    k, dout, dstate = case([2500, 40, 1200], 70, 1, N, F32)
    ref = wanted(k, True, dout, dstate)
    y, state = B.spc_selective_scan_forward(**k, want_state=True)
    close(y, ref["y"], F32, "y")
    close(state, ref["state"], F32, "state")
    g = B.spc_selective_scan_backward(dout, **k, dstate=dstate, want_dinitial=True)
    for name in g._fields:
        close(getattr(g, name), ref[name], F32 if name in ("A", "skip", "dt_bias", "initial") else F32, name)


@pytest.mark.parametrize("c,N", [(16, 4), (40, 33)])
def test_many_short_scenes(c, N):
    gen = torch.Generator().manual_seed(2)
    check_all(*case(torch.randint(0, 5, (300,), generator=gen).tolist(), c, 1, N, F32))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("c,G,N", [(64, 1, 16), (1, 1, 1), (130, 2, 8), (65, 1, 3), (90, 3, 17), (20, 1, 64)])
@pytest.mark.parametrize("gate,softplus", [(True, True), (False, False)])
def test_rows_one_by_one(gate, softplus, c, G, N, dtype):
    k, _, _ = case([12] * 5, c, G, N, dtype, gate=gate)
    if not softplus:  # (step sizes above zero: at -7, exp(d A) passes 2^127)
        k["dt"], k["dt_bias"] = (0.05 * k["dt"].abs()).to(dtype), 0.01 * k["dt_bias"].abs()
    ref = wanted(k, softplus)
    at, state = k.pop("offsets"), k.pop("initial_state")
    for t in range(12):
        rows = {n: v[t::12] if n in ("u", "dt", "B", "C", "gate") and v is not None else v for n, v in k.items()}
        y = B.spc_selective_scan_step(rows["u"], rows["dt"], rows["A"], rows["B"], rows["C"], state, rows["skip"], rows["gate"], rows["dt_bias"], softplus=softplus)
        close(y, ref["y"][slice(t, None, 12)], dtype, t)
    close(state, ref["state"], F32, "state")


def test_long_streams_do_not_drift():
    """20 000 rows at a decay of exp(-2^-12) with inputs of 2^-12: each row rounds the state to 24 bits, and the decay itself is no rounding of one."""
    step = torch.full((1, 1), 2.0 ** -12, device="cuda")
    A, one, state = -torch.ones(1, 1, device="cuda"), torch.ones(1, 1, 1, device="cuda"), torch.zeros(1, 1, 1, device="cuda")
    for _ in range(20_000):
        B.spc_selective_scan_step(step * 0 + 1, step, A, one, one, state, softplus=False)
    l = float(torch.exp(torch.tensor(-2.0 ** -12, dtype=torch.float64)))
    ref = 2.0 ** -12 * (1 - l ** 20_000) / (1 - l)
    # (a row adds to a state below 1: roundings of at most 2^-25, remembered for 4096 rows, 1.2e-4 if they all fell one way; chance makes it their root, and ten times that is allowed)
    assert abs(float(state) - ref) <= 10 * 64 * 2.0 ** -25


def test_long_memories():
    """20 000 rows of equal steps, decays l = exp(-1.3 x 2^-12), so 1 / (1 - l) = 3151 rows are remembered.  A row rounds its decay (an exp2 just below 1, a unit of
    2^-24) and the state (2^-24): 2 x 2^-24, all one way at worst.  Segments of L rows (24 here) do that in their own sum and in their outputs, 2 L x 2^-24 each; between them the chain
    does it once a segment, for 3151 / L remembered ones.  4 x 24 + 2 x 3151 / 24 = 359; row by row it could be 2 x 3151."""
    n, d = 20_000, 1.3 * 2.0 ** -12
    d = float(torch.tensor(d, dtype=torch.float32))
    one = torch.ones(n, 1, 1, device="cuda")
    y, state = B.spc_selective_scan_forward(torch.ones(n, 1, device="cuda"), torch.full((n, 1), d, device="cuda"), -torch.ones(1, 1, device="cuda"), one, one, softplus=False, want_state=True)
    l = torch.exp(torch.tensor(-d, dtype=torch.float64))
    t = torch.arange(1, n + 1, dtype=torch.float64)
    ref = d * (1 - l ** t) / (1 - l)
    assert ((y[:, 0].double().cpu() - ref).abs() / ref).max() <= 360 * 2.0 ** -24
    assert abs(float(state) - float(ref[-1])) <= 360 * 2.0 ** -24 * float(ref[-1])


def test_states_carry_on():
    k, dout, _ = case([400], 64, 1, 16, F32)
    y, state = B.spc_selective_scan_forward(**k, want_state=True)
    cut = lambda lo, hi: {n: v[lo:hi] if n in ("u", "dt", "B", "C", "gate") else v for n, v in k.items() if n != "offsets"}  # noqa: E731
    first, middle = B.spc_selective_scan_forward(**cut(0, 150), want_state=True)
    second, last = B.spc_selective_scan_forward(**{**cut(150, 400), "initial_state": middle}, want_state=True)
    ref = wanted(k)
    close(torch.cat([first, second]), ref["y"], F32, "y")
    close(last, ref["state"], F32, "state")


def test_gradients_against_differences():
    k, dout, dstate = case([30, 0, 1, 19], 6, 2, 5, F32)
    g = B.spc_selective_scan_backward(dout, **k, dstate=dstate, want_dinitial=True)
    names = ["u", "dt", "A", "B", "C", "skip", "gate", "dt_bias", "initial_state"]
    gen = torch.Generator().manual_seed(3)

    def loss(v):
        r = wanted({**k, **v})
        return float((r["y"].v * dout.double().cpu()).sum() + (r["state"].v * dstate.double().cpu()).sum())

    for name, grad in zip(names, (g.u, g.dt, g.A, g.B, g.C, g.skip, g.gate, g.dt_bias, g.initial)):
        base = k[name].double()
        d, step = torch.randn(base.shape, generator=gen, dtype=torch.float64).cuda(), 1e-4
        num = (loss({name: base + step * d}) - loss({name: base - step * d})) / (2 * step)
        ana = float((grad.double() * d).sum())
        # (central differences: third derivatives times step^2; fp32 sums of some 300 terms)
        assert abs(num - ana) <= 1e-5 * float((grad.double() * d).abs().sum()), name


@pytest.mark.parametrize("N", [16, 33])
def test_rows_in_no_scene_are_left_alone(N):
    k, dout, dstate = case([90, 0, 60], 70, 1, N, BF16)
    y, state = B.spc_selective_scan_forward(**k, want_state=True)
    g = B.spc_selective_scan_backward(dout, **k, dstate=dstate, want_dinitial=True)
    pad = lambda t: torch.cat([torch.full_like(t[:20], float("nan")), t, torch.full_like(t[:33], float("inf"))])  # noqa: E731
    wide = {n: pad(v) if n in ("u", "dt", "B", "C", "gate") else v for n, v in k.items()} | {"offsets": k["offsets"] + 20}
    out = torch.full((203, 70), 7.0, dtype=BF16, device="cuda")
    _, state2 = B.spc_selective_scan_forward(**wide, want_state=True, out=out)
    outs = [torch.full(s, 7.0, dtype=BF16, device="cuda") for s in ((203, 70), (203, 70), (203, 1, N), (203, 1, N), (203, 70))]
    g2 = B.spc_selective_scan_backward(pad(dout), **wide, dstate=dstate, want_dinitial=True, out=outs)
    for t in (out, *outs):
        assert (t[:20] == 7).all() and (t[170:] == 7).all()
    ref = wanted(k, True, dout, dstate)  # (segments start elsewhere, so not the same bits)
    close(out[20:170], ref["y"], BF16, "y")
    close(state2, ref["state"], F32, "state")
    for name in g2._fields:
        t = getattr(g2, name)
        close(t[20:170] if t.shape[0] == 203 else t, ref[name], BF16 if t.dtype == BF16 else F32, name)


def test_no_rows():
    k, dout, dstate = case([0, 0], 20, 1, 16, F16)
    y, state = B.spc_selective_scan_forward(**k, want_state=True)
    assert y.shape == (0, 20) and torch.equal(state, k["initial_state"])
    g = B.spc_selective_scan_backward(dout, **k, dstate=dstate, want_dinitial=True)
    assert torch.equal(g.initial, dstate) and all((t == 0).all() for t in (g.A, g.skip, g.dt_bias))
    assert B.spc_selective_scan_step(k["u"], k["dt"], k["A"], k["B"], k["C"], state[:0]).shape == (0, 20)


def test_infinities_and_nan_reach_later_rows_of_their_scene_only():
    k, dout, _ = case([100, 80], 130, 2, 16, F32, states=False)
    y, _ = B.spc_selective_scan_forward(**k)
    for name, index, later in (("u", (40, 3), lambda m: m[40:100, 3:4]), ("B", (40, 1, 5), lambda m: m[40:100, 65:]), ("gate", (99, 7), lambda m: m[99:100, 7:8]),
                               ("dt", (120, 129), lambda m: m[120:, 129:])):
        for value in (float("nan"), float("inf")):
            t = k[name].clone()
            t[index] = value
            y2, _ = B.spc_selective_scan_forward(**{**k, name: t})
            touched = torch.zeros_like(y, dtype=torch.bool)
            later(touched)[:] = True
            assert torch.equal(y2[~touched], y[~touched]), (name, value)
            assert not torch.isfinite(y2[touched][0])
    # gradients: rows of the other scene, and other channels' du, have nothing of it
    g = B.spc_selective_scan_backward(dout, **k)
    bad = dout.clone()
    bad[40, 3] = float("nan")
    g2 = B.spc_selective_scan_backward(bad, **k)
    for name in ("u", "dt", "gate"):
        a, b = getattr(g, name), getattr(g2, name)
        assert torch.equal(a[100:], b[100:]) and torch.equal(a[41:], b[41:]) and torch.equal(a[:, 4:], b[:, 4:]) and torch.isnan(getattr(g2, "u")[:41, 3]).all()
    for a, b in ((g.B, g2.B), (g.C, g2.C)):
        assert torch.equal(a[41:], b[41:]) and torch.equal(a[:, 1], b[:, 1])


def test_shared_inputs_of_no_pitch():
    """B and C the same in every row: their gradients come row by row."""
    k, dout, dstate = case([120, 30], 64, 2, 16, F16)
    k["B"], k["C"] = k["B"][:1].expand(150, 2, 16), k["C"][3:4, :1].expand(150, 2, 16)
    check_all(k, dout, dstate)


def test_recorded_beside_eager_calls_on_other_streams():
    k, dout, dstate = case([1500, 700], 128, 1, 16, BF16)

    def step():
        y, state = B.spc_selective_scan_forward(**k, want_state=True)
        return (y, state, *B.spc_selective_scan_backward(dout, **k, dstate=dstate, want_dinitial=True))

    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    graphs = []
    for _ in range(2):  # two graphs of the same calls, whose scratch is not to be shared with what runs between replays
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            graphs.append((step(), graph))
    for _ in range(3):
        k["u"].normal_()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            eager = step()
        for out, graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for out, _ in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all(torch.equal(a, b) for a, b in zip(eager, want))


def spread(n, c, dtype, gen):
    """-150 to 150 in even steps, in any order."""
    return torch.linspace(-150, 150, n * c, dtype=torch.float64)[torch.randperm(n * c, generator=gen)].view(n, c).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("which", ["gate", "dt"])
def test_gates_and_steps_far_from_zero(which, dtype):
    """exp(-gate) passes 2^128 at -88.7; steps of dt are exp(dt) below, dt above."""
    gen = torch.Generator().manual_seed(8)
    k, dout, dstate = case([200, 0, 100], 64, 1, 5, dtype)
    k[which] = spread(300, 64, dtype, gen)
    check_all(k, dout, dstate)
    k, _, _ = case([1] * 300, 64, 1, 5, dtype)
    k[which] = spread(300, 64, dtype, gen)
    ref = wanted(k)
    state = k["initial_state"]
    y = B.spc_selective_scan_step(k["u"], k["dt"], k["A"], k["B"], k["C"], state, k["skip"], k["gate"], k["dt_bias"])
    close(y, ref["y"], dtype, "y")
    close(state, ref["state"], F32, "state")


def many_scenes(n, scenes, c, N, gen):
    """One long scene and many of a few rows; no decays, steps of one, whole numbers: every sum is exact."""
    cuts = torch.randint(n - 4000, n + 1, (scenes - 1,), generator=gen).sort().values
    at = torch.cat([torch.zeros(1, dtype=torch.long), cuts, torch.tensor([n])]).to(torch.int32).cuda()
    one = torch.zeros(1, 1, N, device="cuda")
    one[..., 3] = 1
    u = torch.randint(-1, 2, (n, c), generator=torch.Generator("cuda").manual_seed(9), device="cuda").float()
    k = {"u": u, "dt": torch.ones(n, c, device="cuda"), "A": torch.zeros(c, N, device="cuda"), "B": torch.ones(1, 1, N, device="cuda").expand(n, 1, N),
         "C": one.expand(n, 1, N), "offsets": at}
    scene = torch.searchsorted(at[1:].contiguous(), torch.arange(n, dtype=torch.int32, device="cuda"), right=True)
    return k, at.long(), scene


def test_chains_of_many_scenes():
    """5000 scenes of 1024 channels of 64 states: sixteen waves for each 64 of their states would pass the 2^32 threads of a launch."""
    k, at, scene = many_scenes(120_000, 5000, 1024, 64, torch.Generator().manual_seed(1))
    y, _ = B.spc_selective_scan_forward(**k, softplus=False)
    for c0 in range(0, 1024, 128):
        total = torch.cat([torch.zeros(1, 128, dtype=torch.float64, device="cuda"), k["u"][:, c0:c0 + 128].double().cumsum(0)])
        assert torch.equal(y[:, c0:c0 + 128].double(), total[1:] - total[at[scene]])


def test_gradients_chains_of_many_scenes():
    """34 900 scenes of 960 channels of 16 states: nine waves, both ways."""
    k, at, scene = many_scenes(120_000, 34_900, 960, 16, torch.Generator().manual_seed(2))
    dout = torch.randint(-1, 2, (120_000, 960), generator=torch.Generator("cuda").manual_seed(5), device="cuda").float()
    g = B.spc_selective_scan_backward(dout, **k, softplus=False)
    db = 0
    for c0 in range(0, 960, 192):
        total = torch.cat([torch.zeros(1, 192, dtype=torch.float64, device="cuda"), dout[:, c0:c0 + 192].double().cumsum(0)])
        q = total[at[scene + 1]] - total[:-1]
        u = k["u"][:, c0:c0 + 192].double()
        assert torch.equal(g.u[:, c0:c0 + 192].double(), q) and torch.equal(g.dt[:, c0:c0 + 192].double(), q * u)
        db = db + (q * u).sum(1)
    assert torch.equal(g.B[:, 0, 3].double(), db)


def check_growing(k, dout, dstate):
    k["dt_bias"] = None
    check_all(k, dout, dstate, softplus=False)


@pytest.mark.parametrize("lengths,c,N,rate,few", [([9000, 20], 5, 3, 1.2, 40), ([9000, 20], 3, 3, 8.0, 8), ([200, 3], 66, 2, 15.0, 5), ([300, 3], 3, 40, 15.0, 5)])
def test_growing_states_stay_zero_until_an_input(lengths, c, N, rate, few):
    """exp(d A) above one: what is zero stays zero, forward until the scene's last rows, backward behind its first ones, though the rows between would grow beyond 2^128."""
    k, dout, dstate = case(lengths, c, 1, N, F32)
    n = lengths[0]
    k["A"] = torch.linspace(0.1, 1.0, c * N, device="cuda").view(c, N) * rate
    k["A"][:, 1] *= -1
    k["dt"] = torch.ones_like(k["dt"])
    k["dt"][n:] = 0.1
    k["u"][:n - few] = 0
    dout[few:n] = 0
    k["initial_state"][0], dstate[0] = 0, 0
    check_growing(k, dout, dstate)


def test_growing_states_of_little():
    """States of 1e-36 that grow by exp(160), both ways: the powers pass 2^128, the states do not."""
    k, dout, dstate = case([20], 70, 1, 5, F32)
    k["A"], k["dt"] = torch.full_like(k["A"], 8.0), torch.ones_like(k["dt"])
    k["u"].zero_()
    k["initial_state"] *= 1e-36
    dstate *= 1e-36
    dout[:18], dout[18:] = 0, 1e-36 * dout[18:]
    check_growing(k, dout, dstate)


def test_steps_of_both_signs():
    """Steps of 10 in rows 32 to 43, of -8 in rows 44 to 53: decays of exp(-120) that rows of exp(80) follow.  A gradient that comes from behind grows first and decays then."""
    k, dout, dstate = case([9000], 3, 1, 2, F32, gate=False, states=False, skip=False)
    k["A"], k["dt"] = torch.tensor([[-1.0, -0.9]] * 3, device="cuda"), torch.full_like(k["dt"], 0.01)
    k["dt"][32:44], k["dt"][44:54] = 10, -8
    k["u"][:44] = 0
    dout[:54], dout[64:] = 0, 0
    check_growing(k, dout, dstate)


@pytest.mark.parametrize("c,N", [(20, 5), (3, 40)])
def test_long_chains(c, N):
    """More than 800 segments in a scene, both ways, so that every wave of a chain has more than one batch of 32; a short scene beside it."""
    check_all(*case([40_000, 50], c, 1, N, F32))
