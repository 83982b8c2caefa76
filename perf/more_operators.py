"""Measured cases of the operators of a selective state space block over sorted voxels: root-mean-square norm with a residual (16 and 8-bit
outputs, gradients), the 1x1x1 product of 8-bit rows, the short causal convolution and the selective scan (each forward and backward),
and one more row of many streams through the last two.

Rows are voxels in sorted order, scenes lie one behind the other, and `offsets` holds the first row of each.  Inputs are column ranges of
projections' outputs where a block would have them so.  Sizes are those of the library's clouds and levels (2 k to 240 k voxels, 16 to 256
channels, twice as many inside the block), with 16 states to a channel.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_F8 = torch.float8_e4m3fn
_F8_MOST = 448.0
_EPS = 1e-5


def _rms(name, op, n, c, dtype, extra=False, pitched=False):
    """extra: forward with a residual, backward with a gradient that reaches the sum past the norm; pitched: rows of a wider buffer."""
    return {"name": name, "op": op, "n": n, "c": c, "dtype": dtype, "extra": extra, "pitched": pitched}


def _linear(name, n, c, cout, dtype):
    return {"name": name, "op": "linear8", "n": n, "c": c, "cout": cout, "dtype": dtype}


def _conv(name, op, n, c, width, dtype, scenes=1, states=False, pitched=False):
    """states: forward from and to the rows in front of the scenes, backward with a gradient of the last ones."""
    return {"name": name, "op": op, "n": n, "c": c, "width": width, "dtype": dtype, "scenes": scenes, "states": states, "pitched": pitched}


def _scan(name, op, n, c, states_n, dtype, groups=1, gate=True, scenes=1, states=False):
    return {"name": name, "op": op, "n": n, "c": c, "N": states_n, "groups": groups, "dtype": dtype, "gate": gate, "scenes": scenes, "states": states}


def listed():
    return [
        # rows of a small cloud in fp32: an object crop, a unit test of a user's model
        _rms("rms_tiny_f32", "rms", 2118, 64, "f32"),
        # pre-norm of a served block on one LiDAR cloud: the residual added, the projection's input in 8 bits
        _rms("rms_quant_lidar", "rms_quant", 120_000, 256, "bf16", extra=True),
        # four indoor scans in training, with the gradient of the residual branch
        _rms("rms_grad_indoor", "rms_grad", 240_000, 256, "bf16", extra=True),
        # the block's first projection served in 8 bits, on a coarse level and on a LiDAR cloud
        _linear("linear8_coarse", 6011, 128, 512, "bf16"),
        _linear("linear8_lidar", 120_000, 256, 1024, "f16"),
        # one LiDAR cloud, one long sequence, the convolution's input half of a projection's columns
        _conv("conv_lidar", "conv", 120_000, 512, 4, "bf16", pitched=True),
        # channels that are no multiple of a vector, seven scenes, one of them empty, carried on from rows before
        _conv("conv_grad_ragged", "conv_grad", 70_001, 90, 3, "f16", scenes=7, states=True),
        # the smallest scan: a small cloud in fp32
        _scan("scan_tiny_f32", "scan", 2118, 64, 16, "f32", gate=False),
        # one LiDAR cloud
        _scan("scan_lidar", "scan", 120_000, 512, 16, "bf16"),
        # a coarse level in training, two scenes carried on from states
        _scan("scan_grad_coarse", "scan_grad", 6011, 256, 16, "bf16", scenes=2, states=True),
        # training on a LiDAR cloud
        _scan("scan_grad_lidar", "scan_grad", 120_000, 512, 16, "bf16"),
        # many streams served together, a row of each: the convolution and the scan behind it
        {"name": "step_many", "op": "step", "n": 2048, "c": 512, "N": 16, "groups": 1, "width": 4, "dtype": "f16", "gate": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    flops = max(work(c)["flops"] for c in listed() if c["op"] != "linear8")
    products = max(work(c)["flops"] for c in listed() if c["op"] == "linear8")
    while True:
        op = rng.choice(["rms", "rms_quant", "rms_grad", "linear8", "conv", "conv_grad", "scan", "scan", "scan_grad", "scan_grad", "step"])
        c = {"op": op, "dtype": rng.choice(["f16", "bf16", "bf16", "f32"]), "n": _log_int(rng, 1000, 240_000)}
        if op in ("rms", "rms_quant", "rms_grad"):
            c["c"] = rng.choice([16, 24, 32, 40, 64, 96, 128, 192, 256, 384, 512, 1024, _log_int(rng, 5, 600)])
            c["extra"], c["pitched"] = rng.random() < 0.5, rng.random() < 0.25
        elif op == "linear8":
            c["c"] = rng.choice([16, 32, 48, 64, 128, 192, 256, 512, _log_int(rng, 5, 512)])
            c["cout"] = rng.choice([32, 64, 128, 256, 384, 512, 1024, _log_int(rng, 5, 1024)])
        elif op in ("conv", "conv_grad"):
            c["c"] = rng.choice([16, 32, 48, 64, 128, 256, 384, 512, 1024, _log_int(rng, 5, 600)])
            c["width"], c["scenes"] = rng.choice([2, 3, 4, 4]), rng.choice([1, 1, 2, 4, 7])
            c["states"], c["pitched"] = rng.random() < 0.4, rng.random() < 0.4
        else:
            c["groups"] = rng.choice([1, 1, 1, 2, 4])
            c["c"] = c["groups"] * rng.choice([16, 32, 48, 64, 128, 128, 256, 256, 512, _log_int(rng, 5, 300)])
            c["N"] = rng.choice([4, 8, 16, 16, 16, 32, _log_int(rng, 1, 32)])
            c["gate"] = rng.random() < 0.6
            if op == "step":
                c["n"], c["width"] = _log_int(rng, 1, 4096), rng.choice([2, 3, 4])
            else:
                c["scenes"], c["states"] = rng.choice([1, 1, 2, 4, 7]), rng.random() < 0.4
        w = work(c)
        if w["bytes"] <= most and w["flops"] <= (products if op == "linear8" else flops):
            return c


# ---------------------------------------------------------------- inputs
def _lengths(case, seed):
    """Rows of every scene: unlike ones, one of them empty from seven scenes on."""
    n, b = case["n"], case["scenes"]
    gen = torch.Generator().manual_seed(seed)
    share = torch.rand(b, generator=gen) + 0.25
    if b >= 7:
        share[b // 2] = 0.0
    cut = (torch.cumsum(share, 0) / share.sum() * n).floor().long()
    cut[-1] = n
    return torch.diff(cut, prepend=torch.zeros(1, dtype=torch.long))


def _as_f8(t):
    """(e4m3 rows, their scales) of rows in 32 bits."""
    scale = t.abs().amax(1) / _F8_MOST
    return (t / scale[:, None]).clamp(-_F8_MOST, _F8_MOST).to(_F8), scale


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt, op, n, c = _DTYPES[case["dtype"]], case["op"], case["n"], case["c"]

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    def unit(*shape):
        return torch.rand(*shape, generator=gen, device=dev)

    def rows(t, wide):
        if not wide:
            return t.to(dt)
        both = torch.zeros(n, 2 * c, dtype=dt, device=dev)
        both[:, :c] = t
        return both[:, :c]

    s = {"op": op, "dtype": dt}
    if op in ("rms", "rms_quant", "rms_grad"):
        spread = 0.5 + 1.5 * unit(c)  # features after a layer: channels of unlike spread and level
        s |= {"x": rows(rand(n, c) * spread + 0.7 * rand(c), case["pitched"]), "gamma": 1 + 0.2 * rand(c),
              "extra": rows(rand(n, c), case["pitched"]) if case["extra"] else None}
        if op == "rms_grad":
            s["rstd"] = (s["x"].float().square().mean(1) + _EPS).rsqrt()
            s["dy"] = rows(rand(n, c), case["pitched"])
        return s
    if op == "linear8":
        s["x"], s["x_scale"] = _as_f8(rand(n, c) * (0.5 + 1.5 * unit(c)))
        s["w"], s["w_scale"] = _as_f8(rand(case["cout"], c) * c ** -0.5)
        return s
    if op != "step":
        lengths = _lengths(case, seed)
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(lengths, 0)]).to(torch.int32).to(dev)
        s["longest"] = int(lengths.max())
        b = case["scenes"]
    if op in ("conv", "conv_grad", "step"):
        w = case["width"]
        s |= {"x": rows(rand(n, c), case.get("pitched", True)), "weight": rand(c, w) * w ** -0.5, "bias": 0.1 * rand(c)}
        if op == "step":
            s["past"] = rand(n, w - 1, c).to(dt)
        else:
            s["past"] = rand(b, w - 1, c).to(dt) if case["states"] else None
        if op == "conv_grad":
            s["dy"] = rand(n, c).to(dt)
            s["dpast"] = rand(b, w - 1, c).to(dt) if case["states"] else None
        if op != "step":
            return s
    N, G = case["N"], case["groups"]
    # rates of -1 to -N, steps of 1e-3 to 0.1 where the projection gives nothing: memories of a few rows to a thousand
    s["A"] = -torch.arange(1, N + 1, device=dev) * torch.exp(0.1 * rand(c, N))
    step = torch.exp(math.log(1e-3) + unit(c) * math.log(100.0))
    s["dt_bias"] = step + torch.log(-torch.expm1(-step))
    s["skip"] = 1 + 0.2 * rand(c)
    if op != "step":
        v = rand(n, c)
        s["u"] = (v * torch.sigmoid(v)).to(dt)
    s["dt"] = (0.5 * rand(n, c)).to(dt)
    low = rand(n, 16 + 2 * G * N).to(dt)  # a projection's output: what the steps are made of, B, C
    s["B"], s["C"] = low[:, 16:16 + G * N].unflatten(1, (G, N)), low[:, 16 + G * N:].unflatten(1, (G, N))
    s["gate"] = rand(n, 2 * c).to(dt)[:, c:] if case["gate"] else None
    if op == "step":
        s["state"] = rand(n, c, N)
        return s
    s["initial"] = rand(b, c, N) if case["states"] else None
    if op == "scan_grad":
        s["dout"] = rand(n, c).to(dt)
        s["dlast"] = 0.1 * rand(b, c, N) if case["states"] else None
    return s


# ---------------------------------------------------------------- the plain form
def _silu(t):
    return t / (1 + torch.exp(-t))


def _silu_slope(t):
    p = 1 / (1 + torch.exp(-t))
    return p * (1 + t * (1 - p))


def _softplus(t):
    return t.clamp(min=0) + torch.log1p(torch.exp(-t.abs()))


def _plain_rms(s):
    z = s["x"].float()
    if s["extra"] is not None:
        z = z + s["extra"].float()
    rstd = (z.square().mean(1) + _EPS).rsqrt()
    y = z * rstd[:, None] * s["gamma"]
    out = {"rstd": rstd}
    if s["op"] == "rms":
        out["y"] = y.to(s["dtype"])
    else:
        out["q"], out["scale"] = _as_f8(y)
    if s["extra"] is not None:
        out["sum"] = z.to(s["dtype"])
    return out


def _plain_rms_grad(s):
    h = s["x"].float() * s["rstd"][:, None]
    dy = s["dy"].float()
    w = dy * s["gamma"]
    dx = s["rstd"][:, None] * (w - h * (w * h).mean(1, keepdim=True))
    if s["extra"] is not None:
        dx = dx + s["extra"].float()
    return {"dx": dx.to(s["dtype"]), "dgamma": (dy * h).sum(0, dtype=torch.float64).float()}


def _plain_linear8(s):
    return {"y": (torch.mm(s["x"].float(), s["w"].float().t()) * s["x_scale"][:, None] * s["w_scale"]).to(s["dtype"])}


def _scenes(s, n):
    """(scene, row in it, rows behind it) of every row; the scenes' first rows and ends."""
    first, end = s["offsets"][:-1].long(), s["offsets"][1:].long()
    scene = torch.repeat_interleave(torch.arange(len(first), device=first.device), end - first, output_size=n)
    row = torch.arange(n, device=first.device)
    return scene, row - first[scene], end[scene] - 1 - row, first, end


def _window(s, x, past, scene, at):
    """Row t - k of every row t, k = 0 .. width - 1."""
    row, w = torch.arange(x.shape[0], device=x.device), s["weight"].shape[1]

    def back(k):
        v = torch.where((at >= k)[:, None], x[(row - k).clamp(min=0)], 0)
        return v if past is None or k == 0 else torch.where((at >= k)[:, None], v, past[scene, (w - 1 - k + at).clamp(max=w - 2)])

    return [back(k) for k in range(w)]


def _plain_conv(s):
    x, weight = s["x"].float(), s["weight"]
    n, w = x.shape[0], weight.shape[1]
    past = None if s["past"] is None else s["past"].float()
    scene, at, _, first, end = _scenes(s, n)
    rows = _window(s, x, past, scene, at)
    pre = s["bias"] + sum(weight[:, w - 1 - k] * rows[k] for k in range(w))
    if s["op"] == "conv":
        out = {"y": _silu(pre).to(s["dtype"])}
        if past is not None:
            back, length = torch.arange(w - 1, 0, -1, device=x.device), (end - first)[:, None]
            kept = x[(end[:, None] - back).clamp(0, n - 1)]
            older = torch.gather(past, 1, (w - 1 - back + length).clamp(max=w - 2)[..., None].expand(-1, -1, x.shape[1]))
            out["past"] = torch.where((length >= back)[..., None], kept, older).to(s["dtype"])
        return out
    dpre = s["dy"].float() * _silu_slope(pre)
    left = (end - first)[scene] - 1 - at
    row = torch.arange(n, device=x.device)
    dx = sum(weight[:, w - 1 - k] * torch.where((left >= k)[:, None], dpre[(row + k).clamp(max=n - 1)], 0) for k in range(w))
    out = {"dweight": torch.stack([(dpre * rows[w - 1 - j]).sum(0, dtype=torch.float64).float() for j in range(w)], 1),
           "dbias": dpre.sum(0, dtype=torch.float64).float()}
    if past is not None:
        dpast = s["dpast"].float()
        dx = dx + torch.where((left < w - 1)[:, None], dpast[scene, (w - 2 - left).clamp(min=0)], 0)
        # row i of the state is row i - (w - 1) of the scene: read by rows that lie k behind it, kept where the scene is shorter than that
        i, length = torch.arange(w - 1, device=x.device), (end - first)[:, None]

        def read(k):
            t = i - (w - 1) + k
            return torch.where(((t >= 0) & (t < length))[..., None], weight[:, w - 1 - k] * dpre[(first[:, None] + t).clamp(0, n - 1)], 0)

        dstate = sum(read(k) for k in range(w))
        stays = i - length
        dstate = dstate + torch.where((stays >= 0)[..., None], torch.gather(dpast, 1, stays.clamp(min=0)[..., None].expand(-1, -1, x.shape[1])), 0)
        out["dinitial"] = dstate.to(s["dtype"])
    return out | {"dx": dx.to(s["dtype"])}


def _steps(s):
    """What the scan's rows are made of: step sizes, decays, inputs, B and C of every channel."""
    c, G = s["A"].shape[0], s["B"].shape[1]
    wide = lambda t: t.float().repeat_interleave(c // G, 1)  # noqa: E731
    x = s["dt"].float() + s["dt_bias"]
    delta = _softplus(x)
    return x, delta, torch.exp(delta[..., None] * s["A"]), (delta * s["u"].float())[..., None] * wide(s["B"]), wide(s["C"]), wide(s["B"])


def _along(coef, more, longest):
    """v_t = coef_t v_{t-1} + more_t of all rows at once, by doubling (coef is zero in the first row of every scene); in place."""
    s = 1
    while s < longest:
        more[s:] += coef[s:] * more[:-s]
        coef[s:] = coef[s:] * coef[:-s]
        s *= 2
    return more


def _states(s, a, bx, first, some):
    """h of every row."""
    coef, more = a.clone(), bx
    if s["initial"] is not None:
        more[first[some]] += a[first[some]] * s["initial"][some]
    coef[first[some]] = 0
    return _along(coef, more, s["longest"])


def _plain_scan(s):
    n = s["dt"].shape[0]
    _, _, _, first, end = _scenes(s, n)
    some = end > first
    _, _, a, bx, C, _ = _steps(s)
    h = _states(s, a, bx, first, some)
    y = (h * C).sum(2) + s["skip"] * s["u"].float()
    if s["gate"] is not None:
        y = y * _silu(s["gate"].float())
    out = {"y": y.to(s["dtype"])}
    if s["initial"] is not None:
        out["state"] = torch.where(some[:, None, None], h[(end - 1).clamp(min=0)], s["initial"])
    return out


def _plain_scan_grad(s):
    n, G = s["dt"].shape[0], s["B"].shape[1]
    _, _, _, first, end = _scenes(s, n)
    some = end > first
    x, delta, a, bx, C, B = _steps(s)
    u, dout = s["u"].float(), s["dout"].float()
    h = _states(s, a, bx, first, some)
    out = {}
    dy = dout
    if s["gate"] is not None:
        gate = s["gate"].float()
        y = (h * C).sum(2) + s["skip"] * u
        out["dgate"] = (dout * y * _silu_slope(gate)).to(s["dtype"])
        dy = dout * _silu(gate)
    out["dC"] = (h * dy[..., None]).unflatten(1, (G, -1)).sum(2).to(s["dtype"])
    g = C * dy[..., None]
    if s["initial"] is not None:
        g[end[some] - 1] += s["dlast"][some]
    behind = torch.cat([a[1:], torch.zeros_like(a[:1])])  # the decay between a row and the next
    behind[end[some] - 1] = 0
    g = torch.flip(_along(torch.flip(behind, [0]), torch.flip(g, [0]), s["longest"]), [0])
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[first[some]] = 0 if s["initial"] is None else s["initial"][some]
    dlog = g * a * before
    dxu = (g * B).sum(2)
    ddelta = u * dxu + (dlog * s["A"]).sum(2)
    ddt = ddelta / (1 + torch.exp(-x))
    out |= {"du": (delta * dxu + s["skip"] * dy).to(s["dtype"]), "ddt": ddt.to(s["dtype"]),
            "dA": (dlog * delta[..., None]).sum(0, dtype=torch.float64).float(),
            "dB": (g * (delta * u)[..., None]).unflatten(1, (G, -1)).sum(2).to(s["dtype"]),
            "dskip": (dy * u).sum(0, dtype=torch.float64).float(), "dbias": ddt.sum(0, dtype=torch.float64).float()}
    if s["initial"] is not None:
        at = first.clamp(max=n - 1)
        out["dinitial"] = torch.where(some[:, None, None], a[at] * g[at], s["dlast"])
    return out


def _plain_step(s):
    w, dt = s["weight"].shape[1], s["dtype"]
    rows = torch.cat([s["past"], s["x"][:, None]], 1)
    u = _silu(s["bias"] + (rows.float() * s["weight"].t()).sum(1)).to(dt)
    s["past"].copy_(rows[:, 1:])
    _, _, a, bx, C, _ = _steps(s | {"u": u})
    s["state"].mul_(a).add_(bx)
    y = (s["state"] * C).sum(2) + s["skip"] * u.float()
    if s["gate"] is not None:
        y = y * _silu(s["gate"].float())
    return {"y": y.to(dt), "past": s["past"], "state": s["state"]}


def run(s):
    op = s["op"]
    if not own:
        return {"rms": _plain_rms, "rms_quant": _plain_rms, "rms_grad": _plain_rms_grad, "linear8": _plain_linear8, "conv": _plain_conv,
                "conv_grad": _plain_conv, "scan": _plain_scan, "scan_grad": _plain_scan_grad, "step": _plain_step}[op](s)
    from paper_2511_20834_amd import binding as L

    if op == "rms":
        y, total, rstd = L.spc_rms_norm_forward(s["x"], s["gamma"], eps=_EPS, residual=s["extra"], want_stats=True)
        out = {"y": y, "rstd": rstd}
        return out if total is None else out | {"sum": total}
    if op == "rms_quant":
        q, scale, total, rstd = L.spc_rms_norm_quantize(s["x"], s["gamma"], eps=_EPS, residual=s["extra"], want_stats=True)
        out = {"q": q, "scale": scale, "rstd": rstd}
        return out if total is None else out | {"sum": total}
    if op == "rms_grad":
        dx, dgamma = L.spc_rms_norm_backward(s["dy"], s["x"], s["rstd"], s["gamma"], dsum=s["extra"])
        return {"dx": dx, "dgamma": dgamma}
    if op == "linear8":
        return {"y": L.spc_linear_f8(s["x"], s["x_scale"], s["w"], s["w_scale"], dtype=s["dtype"])}
    if op == "conv":
        y, past = L.spc_causal_conv_forward(s["x"], s["weight"], s["bias"], s["offsets"], initial_rows=s["past"], want_rows=s["past"] is not None)
        return {"y": y} if past is None else {"y": y, "past": past}
    if op == "conv_grad":
        dx, dweight, dbias, dinitial = L.spc_causal_conv_backward(s["dy"], s["x"], s["weight"], s["bias"], s["offsets"], initial_rows=s["past"],
                                                                  drows=s["dpast"], want_dinitial=s["past"] is not None)
        out = {"dx": dx, "dweight": dweight, "dbias": dbias}
        return out if dinitial is None else out | {"dinitial": dinitial}
    if op == "step":
        u = L.spc_causal_conv_step(s["x"], s["weight"], s["past"], s["bias"])
        y = L.spc_selective_scan_step(u, s["dt"], s["A"], s["B"], s["C"], s["state"], skip=s["skip"], gate=s["gate"], dt_bias=s["dt_bias"])
        return {"y": y, "past": s["past"], "state": s["state"]}
    if op == "scan":
        y, state = L.spc_selective_scan_forward(s["u"], s["dt"], s["A"], s["B"], s["C"], skip=s["skip"], gate=s["gate"], dt_bias=s["dt_bias"],
                                                offsets=s["offsets"], initial_state=s["initial"], want_state=s["initial"] is not None)
        return {"y": y} if state is None else {"y": y, "state": state}
    g = L.spc_selective_scan_backward(s["dout"], s["u"], s["dt"], s["A"], s["B"], s["C"], skip=s["skip"], gate=s["gate"], dt_bias=s["dt_bias"],
                                      offsets=s["offsets"], initial_state=s["initial"], dstate=s["dlast"], want_dinitial=s["initial"] is not None)
    out = {"du": g.u, "ddt": g.dt, "dA": g.A, "dB": g.B, "dC": g.C, "dskip": g.skip, "dbias": g.dt_bias}
    if g.gate is not None:
        out["dgate"] = g.gate
    return out if g.initial is None else out | {"dinitial": g.initial}


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    op, n, c = case["op"], case["n"], case["c"]
    if op in ("rms", "rms_quant"):  # x (and the residual) in, y (and the sum) out, statistics
        y = es if op == "rms" else 1
        return {"bytes": n * (c * (es + y + (2 * es if case["extra"] else 0)) + (4 if op == "rms" else 8)) + 4 * c,
                "flops": n * c * (4 + (1 if case["extra"] else 0) + (3 if op == "rms_quant" else 0))}
    if op == "rms_grad":
        return {"bytes": n * (c * es * (4 if case["extra"] else 3) + 4) + 8 * c, "flops": (10 if case["extra"] else 9) * n * c}
    if op == "linear8":
        m = case["cout"]
        return {"bytes": n * (c + 4) + m * (c + 4) + n * m * es, "flops": 2 * n * c * m}
    if op in ("conv", "conv_grad"):
        w = case["width"]
        past = case["scenes"] * (w - 1) * c * es if case["states"] else 0
        if op == "conv":
            return {"bytes": 2 * n * c * es + 2 * past + 4 * c * (w + 1), "flops": n * c * (2 * w + 5)}
        return {"bytes": 3 * n * c * es + 3 * past + 8 * c * (w + 1), "flops": n * c * (6 * w + 12)}
    N, gates = case["N"], 1 if case["gate"] else 0
    low = 2 * case["groups"] * N * es  # B and C of a row
    params = 4 * c * (N + 2)
    if op == "step":
        w = case["width"]
        return {"bytes": n * (c * es * (3 + gates + 2 * (w - 1)) + low + 8 * c * N) + params + 4 * c * (w + 1), "flops": n * c * (7 * N + 2 * w + 20)}
    state = 4 * case["scenes"] * c * N if case["states"] else 0
    if op == "scan":
        return {"bytes": n * (c * es * (3 + gates) + low) + params + 2 * state, "flops": n * c * (7 * N + 12)}
    return {"bytes": n * (c * es * (5 + 2 * gates) + 2 * low) + 2 * params + 3 * state, "flops": n * c * (22 * N + 30)}


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_conv(case, s, up):
    """A row at a time behind the rows in front of it, scene by scene."""
    w, c, dev = case["width"], case["c"], s["x"].device
    at = s["offsets"].tolist()
    grad = case["op"] == "conv_grad"
    out = {}
    weight = torch.flip(up["weight"], [1]).t()[:, None].contiguous()  # of the row k back

    def act(t):
        p = torch.sigmoid(t)
        return t * p, p + t * p * (1 - p)

    parts = []
    for b, (lo, hi) in enumerate(zip(at, at[1:])):
        past = up["past"][b] if case["states"] else torch.zeros(w - 1, c, dtype=torch.float64, device=dev)
        seq = torch.cat([past, up["x"][lo:hi]])
        m = hi - lo
        pre = up["bias"] + (torch.stack([seq[w - 1 - k:w - 1 - k + m] for k in range(w)]) * weight).sum(0)
        y, slope = act(pre)
        if not grad:
            parts.append({"y": y, "past": seq[m:]})
            continue
        d = up["dy"][lo:hi] * slope
        dseq = torch.zeros_like(seq)
        for k in range(w):
            dseq[w - 1 - k:w - 1 - k + m] += weight[k] * d
        if case["states"]:
            dseq[m:] += up["dpast"][b]
        dw = torch.stack([(d * seq[j:j + m]).sum(0) for j in range(w)], 1)
        parts.append({"dx": dseq[w - 1:], "dinitial": dseq[:w - 1], "dweight": dw, "dbias": d.sum(0)})
    if not grad:
        out["y"] = torch.cat([p["y"] for p in parts])
        if case["states"]:
            out["past"] = torch.stack([p["past"] for p in parts])
        return out
    out = {"dx": torch.cat([p["dx"] for p in parts]), "dweight": sum(p["dweight"] for p in parts), "dbias": sum(p["dbias"] for p in parts)}
    if case["states"]:
        out["dinitial"] = torch.stack([p["dinitial"] for p in parts])
    return out


def _exact_scan(case, s, up):
    """The recurrence a row at a time, forward, and for gradients back again."""
    n, c, N, G = case["n"], case["c"], case["N"], case["groups"]
    dev, grad = s["dt"].device, case["op"] == "scan_grad"
    if n * (2 if grad else 1) > 300_000 or n * c * N * 8 * (3 if grad else 2) > 100e9:
        return None
    at = s["offsets"].tolist()
    starts = {lo: b for b, (lo, hi) in enumerate(zip(at, at[1:])) if hi > lo}
    ends = {hi - 1: b for b, (lo, hi) in enumerate(zip(at, at[1:])) if hi > lo}
    raw = up["dt"] + up["dt_bias"]
    delta = torch.logaddexp(raw, torch.zeros((), dtype=torch.float64, device=dev))
    zero = torch.zeros(c, N, dtype=torch.float64, device=dev)
    spread = lambda t: t.repeat_interleave(c // G, dim=1)  # noqa: E731
    H = torch.empty(n, c, N, dtype=torch.float64, device=dev)
    first = [up["initial"][b] if case["states"] else zero for b in range(case["scenes"])]
    last = [f.clone() for f in first]
    a = torch.empty_like(H)
    for r in range(0, n, 4096):
        e = min(n, r + 4096)
        a[r:e] = torch.exp(delta[r:e, :, None] * up["A"])
        H[r:e] = (delta * up["u"])[r:e, :, None] * spread(up["B"][r:e])
    h = zero
    rows, decays = H.unbind(0), a.unbind(0)
    for t in range(n):
        h = rows[t].addcmul_(decays[t], first[starts[t]] if t in starts else h)
        if t in ends:
            last[ends[t]] = h
    Y = up["skip"] * up["u"]
    for r in range(0, n, 4096):
        e = min(n, r + 4096)
        Y[r:e] += (H[r:e] * spread(up["C"][r:e])).sum(2)
    gate = up["gate"]
    sig = None if gate is None else torch.sigmoid(gate)
    if not grad:
        out = {"y": Y if gate is None else Y * gate * sig}
        return out | {"state": torch.stack(last)} if case["states"] else out
    dout, out = up["dout"], {}
    dy = dout
    if gate is not None:
        out["dgate"] = dout * Y * (sig + gate * sig * (1 - sig))
        dy = dout * gate * sig
    new = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device=dev)  # noqa: E731
    out |= {"dC": new(n, G, N), "dB": new(n, G, N), "dA": new(c, N), "du": up["skip"] * dy, "ddt": new(n, c), "dskip": (dy * up["u"]).sum(0)}
    if case["states"]:
        out["dinitial"] = up["dlast"].clone()
    Q = torch.empty_like(H)  # gradients of the states
    for r in range(0, n, 4096):
        e = min(n, r + 4096)
        Q[r:e] = dy[r:e, :, None] * spread(up["C"][r:e])
    rows, g = Q.unbind(0), None
    for t in range(n - 1, -1, -1):
        if t in ends:
            g = rows[t] if not case["states"] else rows[t].add_(up["dlast"][ends[t]])
        else:
            g = rows[t].addcmul_(decays[t + 1], g)
        if t in starts and case["states"]:
            out["dinitial"][starts[t]] = decays[t] * g
    for r in range(0, n, 4096):
        e = min(n, r + 4096)
        q, d, hh = Q[r:e], delta[r:e], H[r:e]
        x = d * up["u"][r:e]
        out["dC"][r:e] = (hh * dy[r:e, :, None]).view(e - r, G, c // G, N).sum(2)
        out["dB"][r:e] = (q * x[..., None]).view(e - r, G, c // G, N).sum(2)
        dxu = (q * spread(up["B"][r:e])).sum(2)
        passed = q * (hh - x[..., None] * spread(up["B"][r:e]))  # the part of the state that the decay let through
        out["dA"] += (passed * d[..., None]).sum(0)
        out["du"][r:e] += d * dxu
        out["ddt"][r:e] = (up["u"][r:e] * dxu + (passed * up["A"]).sum(2)) * torch.sigmoid(raw[r:e])
    out["dbias"] = out["ddt"].sum(0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    up = {k: t.double() if torch.is_tensor(t) and t.is_floating_point() else t for k, t in s.items()}
    op = case["op"]
    if op in ("rms", "rms_quant"):
        z = up["x"] if up["extra"] is None else up["x"] + up["extra"]
        rstd = 1 / torch.sqrt(torch.einsum("nc,nc->n", z, z) / case["c"] + _EPS)
        y = torch.einsum("nc,n,c->nc", z, rstd, up["gamma"])
        out = {"rstd": rstd}
        if op == "rms":
            out["y"] = y
        else:  # (the values that are rounded to 8 bits)
            top = torch.linalg.vector_norm(y, float("inf"), dim=1)
            out["scale"] = top / _F8_MOST
            out["q"] = y * (_F8_MOST / top)[:, None]
        return out if up["extra"] is None else out | {"sum": z}
    if op == "rms_grad":
        c, r = case["c"], up["rstd"][:, None]
        w = up["dy"] * up["gamma"]
        inner = torch.einsum("nc,nc->n", w, up["x"])[:, None]
        dx = r * w - r ** 3 / c * inner * up["x"]
        return {"dx": dx if up["extra"] is None else dx + up["extra"], "dgamma": torch.einsum("nc,nc,n->c", up["dy"], up["x"], up["rstd"])}
    if op == "linear8":
        x, w = up["x"] * up["x_scale"][:, None], up["w"] * up["w_scale"][:, None]
        return {"y": x @ w.t().contiguous()}
    if op in ("conv", "conv_grad"):
        return _exact_conv(case, s, up)
    if op != "step":
        return _exact_scan(case, s, up)
    G = case["groups"]
    group = torch.arange(case["c"], device=s["x"].device) // (case["c"] // G)
    seq = torch.cat([up["past"], up["x"][:, None]], 1)
    pre = up["bias"] + torch.einsum("bkc,ck->bc", seq, up["weight"])
    u = (pre * torch.sigmoid(pre)).to(s["dtype"]).double()  # (a tensor between two calls, of the rows' type)
    delta = torch.logaddexp(up["dt"] + up["dt_bias"], torch.zeros((), dtype=torch.float64, device=u.device))
    state = torch.exp(delta[..., None] * up["A"]) * up["state"] + (delta * u)[..., None] * up["B"][:, group]
    y = torch.einsum("bcn,bcn->bc", state, up["C"][:, group]) + up["skip"] * u
    return {"y": y if up["gate"] is None else y * up["gate"] * torch.sigmoid(up["gate"]), "past": seq[:, 1:], "state": state}
