"""Measured cases of the operators that mix voxels along the sorted order: layer norm of feature rows and linear attention with a
decay for each head, each forward and backward, and the attention's single-token step.

Rows are voxels in sorted order, scenes lie one behind the other, and `offsets` holds the first row of each.  Queries, keys and values
are column ranges of one projection's output, as a 1x1x1 layer writes it.  Sizes are those of the library's clouds and levels (2 k to
240 k voxels, 16 to 256 channels) in heads of 16 to 128 channels.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-5
_CHUNK = 128  # tokens whose products with each other the plain form takes directly


def _norm(name, op, n, c, dtype, extra=False, pitched=False):
    """extra: forward with a residual, backward with a gradient that reaches the sum past the norm; pitched: rows of a wider buffer."""
    return {"name": name, "op": op, "n": n, "c": c, "dtype": dtype, "extra": extra, "pitched": pitched}


def _attn(name, op, n, heads, kv_heads, dk, dv, dtype, scenes=1, states=False):
    """states: forward from and to a state, backward with a gradient of the last state."""
    return {"name": name, "op": op, "n": n, "heads": heads, "kv_heads": kv_heads, "dk": dk, "dv": dv, "dtype": dtype, "scenes": scenes,
            "states": states}


def listed():
    return [
        # rows of a small cloud in fp32: an object crop, a unit test of a user's model
        _norm("norm_tiny_f32", "norm", 2118, 64, "f32"),
        # pre-norm of a block on one LiDAR cloud, with the residual added on the way
        _norm("norm_lidar", "norm", 120_000, 256, "f16", extra=True),
        # a coarse level in training
        _norm("norm_grad_coarse", "norm_grad", 6011, 128, "bf16"),
        # rows of a channel count that is no multiple of a vector, read out of a wider buffer
        _norm("norm_grad_ragged", "norm_grad", 70_001, 90, "f16", pitched=True),
        # four indoor scans in training, with the gradient of the residual branch
        _norm("norm_grad_indoor", "norm_grad", 240_000, 256, "bf16", extra=True),
        # the smallest mixing call: a small cloud in fp32
        _attn("attention_tiny_f32", "attention", 2118, 4, 4, 16, 16, "f32"),
        # one LiDAR cloud, one long sequence
        _attn("attention_lidar", "attention", 120_000, 8, 8, 64, 64, "f16"),
        # four scenes of unlike lengths, narrow heads, a scene carried on from a state
        _attn("attention_indoor", "attention", 240_000, 4, 4, 32, 32, "bf16", scenes=4, states=True),
        # a coarse level in training, keys and values shared by groups of heads
        _attn("attention_grad_coarse", "attention_grad", 6011, 8, 2, 64, 64, "bf16", scenes=2, states=True),
        # training on a LiDAR cloud
        _attn("attention_grad_lidar", "attention_grad", 120_000, 8, 8, 64, 64, "bf16"),
        # one sensor's stream, a token at a time
        {"name": "step_one", "op": "step", "streams": 1, "heads": 8, "kv_heads": 8, "dk": 64, "dv": 64, "dtype": "bf16"},
        # many streams served together
        {"name": "step_many", "op": "step", "streams": 2048, "heads": 8, "kv_heads": 8, "dk": 64, "dv": 64, "dtype": "f16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    flops = max(work(c)["flops"] for c in listed())
    while True:
        op = rng.choice(["norm", "norm_grad", "attention", "attention", "attention_grad", "attention_grad", "step"])
        c = {"op": op, "dtype": rng.choice(["f16", "bf16", "bf16", "f32"])}
        if op in ("norm", "norm_grad"):
            c["n"] = _log_int(rng, 1000, 400_000)
            c["c"] = rng.choice([16, 24, 32, 40, 64, 96, 128, 192, 256, 384, 512, 1024, _log_int(rng, 5, 600)])
            c["extra"], c["pitched"] = rng.random() < 0.5, rng.random() < 0.25
        else:
            c["heads"] = rng.choice([1, 2, 4, 8, 8, 16])
            c["kv_heads"] = c["heads"] if rng.random() < 0.7 else rng.choice([h for h in (1, 2, 4) if c["heads"] % h == 0])
            c["dk"] = rng.choice([16, 24, 32, 32, 48, 64, 64, 64, 128, _log_int(rng, 5, 128)])
            c["dv"] = c["dk"] if rng.random() < 0.7 else rng.choice([16, 32, 40, 64, 128])
            if op == "step":
                c["streams"] = _log_int(rng, 1, 4096)
            else:
                c["n"] = _log_int(rng, 1000, 240_000)
                c["scenes"] = rng.choice([1, 1, 2, 4, 7])
                c["states"] = rng.random() < 0.4
        w = work(c)
        if w["bytes"] <= most and w["flops"] <= flops:
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


def _decays(heads, dev):
    """ln of 1 - 2^-5 for the first head to 1 - 2^-12 for the last: memories of 32 to 4096 voxels."""
    e = torch.linspace(5.0, 12.0, heads, dtype=torch.float64) if heads > 1 else torch.tensor([8.0], dtype=torch.float64)
    return torch.log1p(-torch.exp2(-e)).float().to(dev)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = _DTYPES[case["dtype"]]

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    if case["op"] in ("norm", "norm_grad"):
        n, c = case["n"], case["c"]
        spread = 0.5 + 1.5 * torch.rand(c, generator=gen, device=dev)  # features after a layer: channels of unlike spread and level
        level = 0.7 * rand(c)

        def rows(t):
            if not case["pitched"]:
                return t.to(dt)
            wide = torch.zeros(n, 2 * c, dtype=dt, device=dev)
            wide[:, :c] = t
            return wide[:, :c]

        s = {"op": case["op"], "x": rows(rand(n, c) * spread + level), "gamma": 1 + 0.2 * rand(c), "beta": 0.1 * rand(c), "extra": None}
        if case["op"] == "norm":
            s["extra"] = rows(rand(n, c)) if case["extra"] else None
            return s
        z = s["x"].float()
        mean = z.mean(1, keepdim=True)
        s["mean"], s["rstd"] = mean[:, 0].contiguous(), ((z - mean).square().mean(1) + _EPS).rsqrt()
        s["dy"] = rows(rand(n, c))
        s["extra"] = rows(rand(n, c)) if case["extra"] else None
        return s
    heads, kv, dk, dv = case["heads"], case["kv_heads"], case["dk"], case["dv"]
    n = case["streams"] if case["op"] == "step" else case["n"]
    qkv = rand(n, heads * dk + kv * dk + kv * dv).to(dt)
    q, k, v = qkv.split([heads * dk, kv * dk, kv * dv], 1)
    s = {"op": case["op"], "q": q.unflatten(1, (heads, dk)), "k": k.unflatten(1, (kv, dk)), "v": v.unflatten(1, (kv, dv)),
         "log_decay": _decays(heads, dev), "scale": dk ** -0.5}
    if case["op"] == "step":
        s["state"] = rand(n, heads, dk, dv)
        return s
    lengths = _lengths(case, seed)
    s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(lengths, 0)]).to(torch.int32).to(dev)
    s["chunks"] = int(((lengths + _CHUNK - 1) // _CHUNK).sum())
    s["initial"] = rand(case["scenes"], heads, dk, dv) if case["states"] else None
    if case["op"] == "attention_grad":
        s["do"] = rand(n, heads, dv).to(dt)
        s["dlast"] = 0.1 * rand(case["scenes"], heads, dk, dv) if case["states"] else None
    return s


# ---------------------------------------------------------------- the plain form
def _plain_norm(s):
    x = s["x"].float()
    z = x if s["extra"] is None else x + s["extra"].float()
    mean = z.mean(1, keepdim=True)
    d = z - mean
    rstd = (d.square().mean(1, keepdim=True) + _EPS).rsqrt()
    out = {"y": (d * rstd * s["gamma"] + s["beta"]).to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if s["extra"] is not None:
        out["sum"] = z.to(s["x"].dtype)
    return out


def _plain_norm_grad(s):
    h = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    w = dy * s["gamma"]
    dx = s["rstd"][:, None] * (w - w.mean(1, keepdim=True) - h * (w * h).mean(1, keepdim=True))
    if s["extra"] is not None:
        dx = dx + s["extra"].float()
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * h).sum(0), "dbeta": dy.sum(0)}


def _plain_scan(x, y, z, log_decay, offsets, chunks, initial=None, reverse=False, shift=1):
    """out_i = sum_{j <= i} l^(i-j) (x_i . y_j) z_j + l^(i+shift) initial^T x_i along every scene (from its end with `reverse`), by chunks:
    products inside a chunk directly, those with earlier chunks through the sums of y z^T.  Also l^(len-1+shift) initial + sum_j l^(len-1-j) y_j z_j^T."""
    dev, C, H = x.device, _CHUNK, log_decay.numel()
    x, y, z = x.float(), y.float(), z.float()
    y, z = y.repeat_interleave(H // y.shape[1], 1), z.repeat_interleave(H // z.shape[1], 1)
    first, end = offsets[:-1].long(), offsets[1:].long()
    count = (end - first + C - 1) // C
    scene = torch.repeat_interleave(torch.arange(len(count), device=dev), count, output_size=chunks)
    at = torch.arange(chunks, device=dev) - (count.cumsum(0) - count)[scene]  # chunk's number in its scene
    pos = at[:, None] * C + torch.arange(C, device=dev)
    length = (end - first)[scene]
    valid = pos < length[:, None]
    row = torch.where(valid, (end[scene][:, None] - 1 - pos) if reverse else first[scene][:, None] + pos, 0)
    X, Y, Z = ((t[row] * valid[:, :, None, None]).transpose(1, 2).contiguous() for t in (x, y, z))  # [chunk, head, C, d]
    i = torch.arange(C, device=dev)

    def power(n):  # l^n for every head, n >= 0
        return torch.exp(log_decay.view(-1, *[1] * n.dim()) * n.clamp(min=0))

    gap = i[:, None] - i
    P = torch.matmul(X, Y.transpose(2, 3).contiguous()) * (power(gap) * (gap >= 0))
    filled = valid.sum(1)
    left = filled[:, None] - 1 - i
    L = torch.matmul((Y * (power(left) * (left >= 0)).transpose(0, 1)[..., None]).transpose(2, 3).contiguous(), Z)  # [chunk, head, dy, dz]
    flat = L.transpose(0, 1).flatten(2)
    same = scene[:, None] == scene
    ahead = at[:, None] - at - 1
    S = torch.matmul(power(ahead * C) * (same & (ahead >= 0)), flat)  # what chunks ahead in the same scene leave at this one's start
    rest = length - at * C - filled
    ends = torch.matmul(power(rest)[:, None] * (scene == torch.arange(len(count), device=dev)[:, None]), flat)
    total = end - first
    S = S.unflatten(2, L.shape[2:]).transpose(0, 1)
    out = torch.matmul(P, Z) + torch.matmul(X, S) * power(i + 1)[None, :, :, None]
    last = ends.unflatten(2, L.shape[2:]).transpose(0, 1)
    if initial is not None:
        out = out + torch.matmul(X, initial[scene]) * power(pos + shift).transpose(0, 1)[..., None]
        last = last + initial * power(torch.where(total > 0, total - 1 + shift, 0)).transpose(0, 1)[..., None, None]
    res = torch.zeros(x.shape[0] + 1, H, z.shape[2], device=dev)
    res[torch.where(valid, row, x.shape[0])] = out.transpose(1, 2)
    return res[:-1], last


def _plain_attention(s):
    o, last = _plain_scan(s["q"], s["k"], s["v"], s["log_decay"], s["offsets"], s["chunks"], s["initial"])
    out = {"o": (s["scale"] * o).to(s["q"].dtype)}
    if s["initial"] is not None:
        out["state"] = last
    return out


def _plain_attention_grad(s):
    dt, scale, kv = s["q"].dtype, s["scale"], s["k"].shape[1]
    g, at, n = s["log_decay"], s["offsets"], s["chunks"]
    H = g.numel()
    k, v = s["k"].repeat_interleave(H // kv, 1), s["v"].repeat_interleave(H // kv, 1)
    start = None if s["initial"] is None else s["initial"].transpose(2, 3).contiguous()
    dq, _ = _plain_scan(s["do"], v, k, g, at, n, start)
    q = s["q"].float() * scale
    dlast = s["dlast"]
    dv, first = _plain_scan(k, q, s["do"], g, at, n, dlast, reverse=True, shift=0)
    dk, _ = _plain_scan(v, s["do"], q, g, at, n, None if dlast is None else dlast.transpose(2, 3).contiguous(), reverse=True, shift=0)
    out = {"dq": (scale * dq).to(dt), "dk": dk.unflatten(1, (kv, H // kv)).sum(2).to(dt), "dv": dv.unflatten(1, (kv, H // kv)).sum(2).to(dt)}
    if dlast is not None:
        some = (at[1:] > at[:-1])[:, None]
        out["dinitial"] = first * torch.where(some, torch.exp(g), 1.0)[..., None, None]
    return out


def _plain_step(s):
    H = s["log_decay"].numel()
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    k, v = k.repeat_interleave(H // k.shape[1], 1), v.repeat_interleave(H // v.shape[1], 1)
    s["state"].mul_(torch.exp(s["log_decay"])[None, :, None, None]).add_(k[..., :, None] * v[..., None, :])
    o = s["scale"] * (q[..., :, None] * s["state"]).sum(2)
    return {"o": o.to(s["q"].dtype), "state": s["state"]}


def run(s):
    if not own:
        return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "attention": _plain_attention, "attention_grad": _plain_attention_grad,
                "step": _plain_step}[s["op"]](s)
    from paper_2511_20834_amd import binding as B

    if s["op"] == "norm":
        y, total, mean, rstd = B.spc_layer_norm_forward(s["x"], s["gamma"], s["beta"], eps=_EPS, residual=s["extra"], want_stats=True)
        out = {"y": y, "mean": mean, "rstd": rstd}
        if total is not None:
            out["sum"] = total
        return out
    if s["op"] == "norm_grad":
        dx, dgamma, dbeta = B.spc_layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], dsum=s["extra"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if s["op"] == "attention":
        o, last = B.spc_linear_attention_forward(s["q"], s["k"], s["v"], s["log_decay"], s["offsets"], scale=s["scale"],
                                                 initial_state=s["initial"], want_state=s["initial"] is not None)
        return {"o": o} if last is None else {"o": o, "state": last}
    if s["op"] == "attention_grad":
        dq, dk, dv, dinitial = B.spc_linear_attention_backward(s["do"], s["q"], s["k"], s["v"], s["log_decay"], s["offsets"], scale=s["scale"],
                                                               initial_state=s["initial"], dstate=s["dlast"],
                                                               want_dinitial=s["initial"] is not None)
        out = {"dq": dq, "dk": dk, "dv": dv}
        if dinitial is not None:
            out["dinitial"] = dinitial
        return out
    o = B.spc_linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], scale=s["scale"])
    return {"o": o, "state": s["state"]}


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":  # x (and the residual) in, y (and the sum) out, statistics
        return {"bytes": case["n"] * (case["c"] * es * (4 if case["extra"] else 2) + 8) + 8 * case["c"],
                "flops": (9 if case["extra"] else 8) * case["n"] * case["c"]}
    if case["op"] == "norm_grad":
        return {"bytes": case["n"] * (case["c"] * es * (4 if case["extra"] else 3) + 8) + 12 * case["c"],
                "flops": (15 if case["extra"] else 14) * case["n"] * case["c"]}
    H, kv, dk, dv = case["heads"], case["kv_heads"], case["dk"], case["dv"]
    rows = es * (H * dk + kv * (dk + dv) + H * dv)  # q, k, v, and o or its gradient
    if case["op"] == "step":
        return {"bytes": case["streams"] * (rows + 8 * H * dk * dv), "flops": 5 * case["streams"] * H * dk * dv}
    states = 4 * case["scenes"] * H * dk * dv if case["states"] else 0
    if case["op"] == "attention":  # a token's outer product and its query's product with the state
        return {"bytes": case["n"] * rows + 2 * states, "flops": 4 * case["n"] * H * dk * dv}
    return {"bytes": case["n"] * (rows + es * (H * dk + kv * (dk + dv))) + 3 * states, "flops": 10 * case["n"] * H * dk * dv}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    up = {k: t.double() if torch.is_tensor(t) and t.is_floating_point() else t for k, t in s.items()}
    if case["op"] == "norm":
        z = up["x"] if up["extra"] is None else up["x"] + up["extra"]
        var, mean = torch.var_mean(z, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + _EPS)
        out = {"y": torch.addcmul(up["beta"], (z - mean[:, None]) * rstd[:, None], up["gamma"]), "mean": mean, "rstd": rstd}
        if up["extra"] is not None:
            out["sum"] = z
        return out
    if case["op"] == "norm_grad":  # the Jacobian's three parts, row by row
        c = case["c"]
        h = (up["x"] - up["mean"][:, None]) * up["rstd"][:, None]
        w = up["dy"] * up["gamma"]
        a, b = w.sum(1, keepdim=True), (w * h).sum(1, keepdim=True)
        dx = up["rstd"][:, None] / c * (c * w - a - h * b)
        if up["extra"] is not None:
            dx = dx + up["extra"]
        return {"dx": dx, "dgamma": torch.einsum("nc,nc->c", up["dy"], h), "dbeta": torch.einsum("nc->c", up["dy"])}
    H, group = case["heads"], case["heads"] // case["kv_heads"]
    g, scale = up["log_decay"], up["scale"]
    if case["op"] == "step":
        o = torch.empty(case["streams"], H, case["dv"], dtype=torch.float64, device=g.device)
        state = torch.empty_like(up["state"])
        for h in range(H):
            kh, vh = up["k"][:, h // group], up["v"][:, h // group]
            state[:, h] = torch.exp(g[h]) * up["state"][:, h] + torch.einsum("ba,bc->bac", kh, vh)
            o[:, h] = scale * torch.einsum("ba,bac->bc", up["q"][:, h], state[:, h])
        return {"o": o, "state": state}
    at = s["offsets"].tolist()
    grad = case["op"] == "attention_grad"
    if sum((b - a) ** 2 for a, b in zip(at, at[1:])) * H * (case["dk"] + case["dv"]) * (2.5 if grad else 1) > 1e14:
        return None
    dev = g.device
    q, k, v, do = up["q"], up["k"], up["v"], up.get("do")
    out = {n: torch.zeros(t.shape, dtype=torch.float64, device=dev) for n, t in ((("dq", q), ("dk", k), ("dv", v)) if grad else ())}
    if not grad:
        out["o"] = torch.zeros(case["n"], H, case["dv"], dtype=torch.float64, device=dev)
    if case["states"]:
        out["dinitial" if grad else "state"] = torch.zeros(case["scenes"], H, case["dk"], case["dv"], dtype=torch.float64, device=dev)
    for b, (lo, hi) in enumerate(zip(at, at[1:])):
        n = hi - lo
        age = torch.arange(n, dtype=torch.float64, device=dev)
        for h in range(H):
            m = h // group
            qh, kh, vh = q[lo:hi, h], k[lo:hi, m].contiguous(), v[lo:hi, m].contiguous()
            decay = torch.exp(g[h] * age)  # l^0 .. l^(n-1)
            if case["states"]:
                S0, whole = up["initial"][b, h], torch.exp(g[h] * n)
                grown = torch.exp(g[h] * (age + 1))[:, None]
                if grad:
                    dS = up["dlast"][b, h]
                    back = torch.flip(decay, [0])[:, None]
                    out["dinitial"][b, h] = whole * dS + scale * (qh * grown).t() @ do[lo:hi, h]
                    out["dk"][lo:hi, m] += back * (vh @ dS.t())
                    out["dv"][lo:hi, m] += back * (kh @ dS)
                    out["dq"][lo:hi, h] += scale * grown * (do[lo:hi, h] @ S0.t())
                else:
                    out["state"][b, h] = whole * S0 + (kh * torch.flip(decay, [0])[:, None]).t() @ vh
                    out["o"][lo:hi, h] += scale * grown * (qh @ S0)
            for r in range(0, n, 2048):  # every pair of a query in [r, e) and a key up to it
                e = min(n, r + 2048)
                gap = age[r:e, None] - age[None, :e]
                W = torch.where(gap >= 0, torch.exp(g[h] * gap.clamp(min=0)), 0.0) * scale
                A = W * (qh[r:e] @ kh[:e].t())
                if not grad:
                    out["o"][lo + r:lo + e, h] += A @ vh[:e]
                    continue
                G = do[lo + r:lo + e, h].contiguous()
                D = W * (G @ vh[:e].t())
                out["dq"][lo + r:lo + e, h] += D @ kh[:e]
                out["dk"][lo:lo + e, m] += D.t() @ qh[r:e]
                out["dv"][lo:lo + e, m] += A.t() @ G
    return out
