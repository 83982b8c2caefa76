"""A block that mixes all voxels of a scene along the sorted order, between sparse convolutions that mix their neighbourhoods:

    y = norm1(x);  q, k, v = y W_qkv;  o = linear attention with decays along every scene;  s = x + o W_out;  z = norm2(s)

The two projections are 1x1x1 layers on the scene's own kernel map, q, k and v the column ranges of one output, and the residual is added
by the second norm.  `forward` takes whole clouds (chunked attention), `backward` gives the gradients of a forward pass, and `begin` / `step`
carry streams of single rows, whose only memory is the attention's state.  Everything runs on the current stream without waiting.

Rows in no scene (in front of offsets[0], or from offsets[-1] on: rejected rows, the rest of a padded buffer) may hold anything, NaN included: nothing of them
reaches other rows or the parameters' gradients.  z and s have no meaning there, x's gradient is zero.  Who knows that there are none says so with `all_rows`."""
from __future__ import annotations

from collections import namedtuple

import torch

from . import binding as B

Saved = namedtuple("Saved", "x y mean1 rstd1 qkv o s mean2 rstd2 offsets kmap inside")
Gradients = namedtuple("Gradients", "x gamma1 beta1 w_qkv w_out gamma2 beta2")


class VoxelMixer:
    def __init__(self, w_qkv, w_out, log_decay, gamma1, beta1, gamma2, beta2, kv_heads=None, eps=1e-5):
        """w_qkv [c, heads * dk + kv_heads * (dk + dv)], w_out [heads * dv, c] of the features' type; log_decay [heads] and the norms' [c]
        fp32.  dk = dv = the heads' share of w_out's rows."""
        self.heads = log_decay.shape[0]
        self.kv_heads = self.heads if kv_heads is None else kv_heads
        self.d = w_out.shape[0] // self.heads
        self.w_qkv, self.w_out, self.log_decay, self.eps = w_qkv, w_out, log_decay, eps
        self.gamma1, self.beta1, self.gamma2, self.beta2 = gamma1, beta1, gamma2, beta2
        self.widths = [self.heads * self.d, self.kv_heads * self.d, self.kv_heads * self.d]
        assert w_out.shape[0] == self.heads * self.d and w_qkv.shape == (w_out.shape[1], sum(self.widths))

    def _split(self, qkv):
        return [t.unflatten(1, (-1, self.d)) for t in qkv.split(self.widths, 1)]

    @staticmethod
    def _project(kmap, x, w):
        return B.spc_conv_forward(kmap, x, w[None], n_out=x.shape[0])

    @staticmethod
    def scenes(keys, desc, n_batch):
        """(kernel map of 1x1x1 layers, first rows of the scenes) of sorted keys: what the blocks of one level share."""
        return B.spc_build_kmap(keys, desc, 1, layout=B.LAYOUT_OS), B.spc_batch_offsets(keys, desc, n_batch)

    def forward(self, x, kmap, offsets, save=False, all_rows=False):
        """x: rows in sorted order; all_rows: every row lies in a scene.  Returns (z, s), and with `save` what backward needs."""
        inside = o = None
        if save and not all_rows and offsets is not None:
            # backward adds up products over all rows, so both factors have to be finite in rows of no scene and one of them zero (us without and with it:
            # 120 k x 256, 8 heads of 64, fp16 705 and 765, backward 4495 and 4618; 2118 x 64, 4 heads of 16, fp32 67 and 110, 156 and 186)
            row = torch.arange(x.shape[0], dtype=torch.int32, device=x.device)
            inside = ((row >= offsets[0]) & (row < offsets[-1]))[:, None]
            x = torch.where(inside, x, 0)
            o = torch.zeros(x.shape[0], self.heads, self.d, dtype=x.dtype, device=x.device)
        y, _, mean1, rstd1 = B.spc_layer_norm_forward(x, self.gamma1, self.beta1, self.eps, want_stats=save)
        qkv = self._project(kmap, y, self.w_qkv)
        o, _ = B.spc_linear_attention_forward(*self._split(qkv), self.log_decay, offsets, out=o)
        o = o.flatten(1)
        z, s, mean2, rstd2 = B.spc_layer_norm_forward(self._project(kmap, o, self.w_out), self.gamma2, self.beta2, self.eps, residual=x,
                                                      want_stats=save)
        return (z, s, Saved(x, y, mean1, rstd1, qkv, o, s, mean2, rstd2, offsets, kmap, inside)) if save else (z, s)

    def backward(self, dz, ds, saved):
        """Gradients for those of z and s (ds may be None).  The weights' are plain products of two tall matrices, in fp32."""
        t = saved
        dqkv = torch.empty_like(t.qkv)
        if t.inside is not None:
            dz, ds = torch.where(t.inside, dz, 0), None if ds is None else torch.where(t.inside, ds, 0)
            dqkv.zero_()
        # the gradient of s goes to the residual and to the projection alike
        g, dgamma2, dbeta2 = B.spc_layer_norm_backward(dz, t.s, t.mean2, t.rstd2, self.gamma2, dsum=ds)
        do = self._project(t.kmap, g, self.w_out.t().contiguous())
        B.spc_linear_attention_backward(do.unflatten(1, (self.heads, self.d)), *self._split(t.qkv), self.log_decay, t.offsets, out=self._split(dqkv))
        dy = self._project(t.kmap, dqkv, self.w_qkv.t().contiguous())
        dx, dgamma1, dbeta1 = B.spc_layer_norm_backward(dy, t.x, t.mean1, t.rstd1, self.gamma1, dsum=g)
        product = lambda a, b: torch.mm(a.float().t().contiguous(), b.float())
        return Gradients(dx, dgamma1, dbeta1, product(t.y, dqkv), product(t.o, g), dgamma2, dbeta2)

    def begin(self, streams):
        """(states of `streams` streams, all zeros, and the kernel map of their rows)."""
        dev = self.w_qkv.device
        rows = torch.arange(streams, dtype=torch.int32, device=dev)  # (sorted keys of as many voxels in a line)
        desc = B.spc_pack_desc_fit([0, 0, 0], [0, 0, max(streams - 1, 0)], 1, 1, 0, 32)
        return torch.zeros(streams, self.heads, self.d, self.d, device=dev), B.spc_build_kmap(rows, desc, 1, layout=B.LAYOUT_OS)

    def step(self, x, state, kmap):
        """One more row x [streams, c] of every stream: (z, s) of it; the states are updated in place."""
        y = B.spc_layer_norm_forward(x, self.gamma1, self.beta1, self.eps)[0]
        o = B.spc_linear_attention_step(*self._split(self._project(kmap, y, self.w_qkv)), self.log_decay, state)
        return B.spc_layer_norm_forward(self._project(kmap, o.flatten(1), self.w_out), self.gamma2, self.beta2, self.eps, residual=x)[:2]
