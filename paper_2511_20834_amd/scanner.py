"""A selective state space block over all voxels of a scene along the sorted order, between sparse convolutions that mix their neighbourhoods:

    s = x (+ residual);  y = rms norm(s);  u, z = y W_in;  u = silu(causal convolution of u);  t, B, C = u W_x;  o = selective scan of u with steps t W_dt, gated by z;
    result = o W_out

The projections are 1x1x1 layers on the scene's own kernel map; u and z, and t, B and C, are the column ranges of one output.  `forward` takes whole clouds and returns (result, s):
the next block adds the two in its norm.  `backward` gives the gradients of a forward pass, `begin` / `step` carry streams of single rows.  A block made by `in_8_bits` is
for serving: its norm writes 8 bits and the first projection, the largest, multiplies in 8 bits.  Everything runs on the current stream without waiting.

Rows in no scene (in front of offsets[0], or from offsets[-1] on: rejected rows, the rest of a padded buffer) may hold anything, NaN included: nothing of them
reaches other rows or the parameters' gradients.  result and s have no meaning there, x's gradient is zero.  Who knows that there are none says so with `all_rows`."""
from __future__ import annotations

from collections import namedtuple

import torch

from . import binding as B
from .mixer import VoxelMixer

Saved = namedtuple("Saved", "s rstd y xz u p dt o offsets kmap inside")
Gradients = namedtuple("Gradients", "x gamma w_in conv_weight conv_bias w_x w_dt dt_bias A skip w_out")


class VoxelScan:
    def __init__(self, gamma, w_in, conv_weight, conv_bias, w_x, w_dt, dt_bias, A, skip, w_out, groups=1, eps=1e-5):
        """w_in [c, 2 d], w_x [d, rank + 2 groups N], w_dt [rank, d], w_out [d, c] of the features' type; gamma [c], conv_weight [d, width], conv_bias, dt_bias and skip
        [d], A [d, N] (below zero) fp32."""
        self.d, self.states = A.shape
        self.rank, self.groups, self.width, self.eps = w_dt.shape[0], groups, conv_weight.shape[1], eps
        self.gamma, self.w_in, self.conv_weight, self.conv_bias, self.w_x, self.w_dt = gamma, w_in, conv_weight, conv_bias, w_x, w_dt
        self.dt_bias, self.A, self.skip, self.w_out = dt_bias, A, skip, w_out
        self.w_in8 = None
        low = groups * self.states
        self.widths = [self.rank, low, low]
        assert w_in.shape[1] == 2 * self.d and w_x.shape == (self.d, self.rank + 2 * low) and w_dt.shape[1] == self.d and w_out.shape == (self.d, w_in.shape[0])

    scenes = staticmethod(VoxelMixer.scenes)
    _project = staticmethod(VoxelMixer._project)

    def in_8_bits(self):
        """The same block for serving, its first projection's weights in 8 bits (a row for each output channel)."""
        m = VoxelScan(self.gamma, self.w_in, self.conv_weight, self.conv_bias, self.w_x, self.w_dt, self.dt_bias, self.A, self.skip, self.w_out, self.groups, self.eps)
        m.w_in8 = B.spc_quantize_rows(self.w_in.t().contiguous())
        return m

    def _low(self, p):
        t, b, c = p.split(self.widths, 1)
        return t, b.unflatten(1, (self.groups, self.states)), c.unflatten(1, (self.groups, self.states))

    def _front(self, x, residual, kmap, want_stats=False):
        """(s, y, rstd, xz): the norm and the first projection."""
        if self.w_in8 is not None:
            assert not want_stats  # (8 bits have no gradients)
            q, scale, s, _ = B.spc_rms_norm_quantize(x, self.gamma, self.eps, residual=residual)
            return x if s is None else s, None, None, B.spc_linear_f8(q, scale, *self.w_in8, dtype=x.dtype)
        y, s, rstd = B.spc_rms_norm_forward(x, self.gamma, self.eps, residual=residual, want_stats=want_stats)
        return x if s is None else s, y, rstd, self._project(kmap, y, self.w_in)

    def forward(self, x, kmap, offsets, residual=None, save=False, all_rows=False):
        """x (and residual): rows in sorted order; all_rows: every row lies in a scene.  Returns (result, s), and with `save` what backward needs."""
        inside = u = o = None
        if save and not all_rows and offsets is not None:
            # backward adds up products over all rows, so both factors have to be finite in rows of no scene and one of them zero (us without and with it: 120 k x 256, 512 channels
            # of 16 states, fp16 965 and 1115, backward 7056 and 7198; 2118 x 64, 128 of 16, fp32 83 and 139, 260 and 307)
            row = torch.arange(x.shape[0], dtype=torch.int32, device=x.device)
            inside = ((row >= offsets[0]) & (row < offsets[-1]))[:, None]
            x, residual = torch.where(inside, x, 0), None if residual is None else torch.where(inside, residual, 0)
            u, o = (torch.zeros(x.shape[0], self.d, dtype=x.dtype, device=x.device) for _ in range(2))
        s, y, rstd, xz = self._front(x, residual, kmap, save)
        u, _ = B.spc_causal_conv_forward(xz[:, :self.d], self.conv_weight, self.conv_bias, offsets, out=u)
        p = self._project(kmap, u, self.w_x)
        t, b, c = self._low(p)
        dt = self._project(kmap, t, self.w_dt)
        o, _ = B.spc_selective_scan_forward(u, dt, self.A, b, c, self.skip, xz[:, self.d:], self.dt_bias, offsets, out=o)
        result = self._project(kmap, o, self.w_out)
        return (result, s, Saved(s, rstd, y, xz, u, p, dt, o, offsets, kmap, inside)) if save else (result, s)

    def backward(self, dresult, ds, saved):
        """Gradients for those of result and s (ds may be None); x's is the residual's too.  The weights' are plain products of two tall matrices, in fp32."""
        t = saved
        dxz, dp, ddt = torch.empty_like(t.xz), torch.empty_like(t.p), torch.empty_like(t.dt)
        du = torch.empty_like(t.u)
        if t.inside is not None:
            dresult, ds = torch.where(t.inside, dresult, 0), None if ds is None else torch.where(t.inside, ds, 0)
            for g in (dxz, dp, ddt, du):
                g.zero_()
        flip = lambda w: w.t().contiguous()  # noqa: E731
        product = lambda a, b: torch.mm(a.float().t().contiguous(), b.float())  # noqa: E731
        do = self._project(t.kmap, dresult, flip(self.w_out))
        low, b, c = self._low(t.p)
        dlow, db, dc = self._low(dp)
        scan = B.spc_selective_scan_backward(do, t.u, t.dt, self.A, b, c, self.skip, t.xz[:, self.d:], self.dt_bias, t.offsets, out=(du, ddt, db, dc, dxz[:, self.d:]))
        B.spc_conv_forward(t.kmap, ddt, flip(self.w_dt)[None], out=dlow)
        du = du + self._project(t.kmap, dp, flip(self.w_x))
        _, dconv, dconv_bias, _ = B.spc_causal_conv_backward(du, t.xz[:, :self.d], self.conv_weight, self.conv_bias, t.offsets, out=dxz[:, :self.d])
        dy = self._project(t.kmap, dxz, flip(self.w_in))
        dx, dgamma = B.spc_rms_norm_backward(dy, t.s, t.rstd, self.gamma, dsum=ds)
        return Gradients(dx, dgamma, product(t.y, dxz), dconv, dconv_bias, product(t.u, dp), product(low, ddt), scan.dt_bias, scan.A, scan.skip, product(t.o, dresult))

    def begin(self, streams):
        """((last rows, states) of `streams` streams, all zeros, and the kernel map of their rows)."""
        dev, dtype = self.w_in.device, self.w_in.dtype
        keys = torch.arange(streams, dtype=torch.int32, device=dev)  # (sorted keys of as many voxels in a line)
        desc = B.spc_pack_desc_fit([0, 0, 0], [0, 0, max(streams - 1, 0)], 1, 1, 0, 32)
        state = torch.zeros(streams, self.width - 1, self.d, dtype=dtype, device=dev), torch.zeros(streams, self.d, self.states, device=dev)
        return state, B.spc_build_kmap(keys, desc, 1, layout=B.LAYOUT_OS)

    def step(self, x, state, kmap, residual=None):
        """One more row x [streams, c] of every stream: (result, s) of it; the state is updated in place."""
        s, _, _, xz = self._front(x, residual, kmap)
        u = B.spc_causal_conv_step(xz[:, :self.d], self.conv_weight, state[0], self.conv_bias)
        t, b, c = self._low(self._project(kmap, u, self.w_x))
        o = B.spc_selective_scan_step(u, self._project(kmap, t, self.w_dt), self.A, b, c, state[1], self.skip, xz[:, self.d:], self.dt_bias)
        return self._project(kmap, o, self.w_out), s
