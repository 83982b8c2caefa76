"""Thin ctypes binding of libspc.so: argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI declared in
``include/spc.h``; PyTorch is used for device memory and streams.  There is no CPU
fallback: loading fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from collections import namedtuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspc.so")

OK = 0
DTYPE_F16, DTYPE_BF16, DTYPE_F32 = 0, 1, 2
LAYOUT_OS, LAYOUT_WS, LAYOUT_BOTH = 1, 2, 3
LAYOUT_WS_SYM = 4  # with LAYOUT_WS: symmetric half-map of a submanifold layer


def LAYOUT_HYBRID_T(t: int) -> int:
    """with LAYOUT_BOTH: build for the hybrid dual dataflow with threshold t (dense offsets in the OS matrix only,
    sparse ones in the WS lists only)."""
    return int(t) << 8


DATAFLOW_OS, DATAFLOW_WS = 0, 1
PACK_VALIDATE = 1
CONV_RELU = 1
CONV_PACKED_WEIGHTS = 2
CONV_OS_PHASE = 4
CONV_OS_SPLITK = 8
CONV_RESIDENT = 16
NET_SEQUENTIAL = 1
NET_PHASE_BARRIER = 2
NET_PIPELINED = 4
ERR_ARG, ERR_RANGE, ERR_DUP, ERR_UNSUPPORTED, ERR_HIP, ERR_NOMEM = -1, -2, -3, -4, -5, -6

EXPORTS = [
    "spc_pack_desc_fit", "spc_pack_coords", "spc_pack_coords_noalloc", "spc_build_kmap", "spc_build_kmap_perm", "spc_build_kmaps_network", "spc_kmap_n_in",
    "spc_kmap_n_out", "spc_kmap_kvol", "spc_kmap_copy_out_keys", "spc_kmap_out_keys", "spc_kmap_in_keys", "spc_kmap_os_map",
    "spc_kmap_ws_lists", "spc_kmap_nnz", "spc_kmap_search_info", "spc_search_count", "spc_resident_count", "spc_kmap_export_triples", "spc_kmap_set_size_hint", "spc_kmap_destroy",
    "spc_conv_forward", "spc_conv_forward_hybrid", "spc_conv_tune_threshold",
    "spc_conv_prepare_weights", "spc_permute_rows",
    "spc_layer_norm_forward", "spc_layer_norm_backward",
    "spc_linear_attention_forward", "spc_linear_attention_backward", "spc_linear_attention_step", "spc_batch_offsets",
    "spc_rms_norm_forward", "spc_rms_norm_quantize", "spc_rms_norm_backward", "spc_quantize_rows", "spc_linear_f8",
    "spc_causal_conv_forward", "spc_causal_conv_backward", "spc_causal_conv_step",
    "spc_selective_scan_forward", "spc_selective_scan_backward", "spc_selective_scan_step",
    "spc_probe_copy", "spc_probe_mfma",
    "spc_release_cache", "spc_last_error", "spc_version",
]


class SpcError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("spc error %d: %s" % (code, msg))
        self.code = code


class PackDesc(ctypes.Structure):
    _fields_ = [("key_bits", ctypes.c_int32), ("bits_b", ctypes.c_int32), ("bits_x", ctypes.c_int32),
                ("bits_y", ctypes.c_int32), ("bits_z", ctypes.c_int32), ("origin", ctypes.c_int32 * 3),
                ("pad", ctypes.c_int32)]

    def as_dict(self):
        return dict(key_bits=self.key_bits, bits_b=self.bits_b, bits_x=self.bits_x, bits_y=self.bits_y,
                    bits_z=self.bits_z, origin=list(self.origin), pad=self.pad)


class LayerDesc(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int32), ("in_stride", ctypes.c_int32), ("layer_stride", ctypes.c_int32),
                ("transposed", ctypes.c_int32), ("layout", ctypes.c_int32)]


class AttnDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_scenes", ctypes.c_int32), ("n_rows", ctypes.c_int64), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("dk", ctypes.c_int32), ("dv", ctypes.c_int32), ("scale", ctypes.c_float)]


class AttnRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_pitch", ctypes.c_int64), ("head_pitch", ctypes.c_int64)]


class ScanDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_scenes", ctypes.c_int32), ("n_rows", ctypes.c_int64), ("channels", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("states", ctypes.c_int32), ("softplus", ctypes.c_int32)]


ScanGradients = namedtuple("ScanGradients", "u dt A B C skip gate dt_bias initial")

_lib = None


def lib():
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("%s is missing: run `python -m paper_2511_20834_amd.build` (or __graft_entry__.build())"
                               % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.spc_pack_desc_fit.argtypes = [ctypes.POINTER(i32), ctypes.POINTER(i32), i32, i32, i32, i32, ctypes.POINTER(PackDesc)]
        L.spc_pack_coords.argtypes = [vp, i64, ctypes.POINTER(PackDesc), vp, vp, vp, ctypes.POINTER(ctypes.c_size_t), i32, vp]
        L.spc_pack_coords_noalloc.argtypes = [vp, i64, ctypes.POINTER(PackDesc), vp, vp, i32, vp]
        L.spc_build_kmap.argtypes = [vp, i64, ctypes.POINTER(PackDesc), ctypes.POINTER(LayerDesc), ctypes.POINTER(vp), vp]
        L.spc_build_kmap_perm.argtypes = [vp, i64, vp, ctypes.POINTER(PackDesc), ctypes.POINTER(LayerDesc), ctypes.POINTER(vp), vp]
        L.spc_build_kmaps_network.argtypes = [vp, i64, ctypes.POINTER(PackDesc), ctypes.POINTER(LayerDesc), i32,
                                              ctypes.POINTER(vp), ctypes.POINTER(vp), i32, i32]
        for f in ("spc_kmap_n_in", "spc_kmap_n_out"):
            getattr(L, f).argtypes = [vp]
            getattr(L, f).restype = i64
        L.spc_kmap_kvol.argtypes = [vp]
        for f in ("spc_kmap_out_keys", "spc_kmap_in_keys", "spc_kmap_os_map"):
            getattr(L, f).argtypes = [vp]
            getattr(L, f).restype = vp
        L.spc_kmap_copy_out_keys.argtypes = [vp, vp, i64]
        L.spc_kmap_ws_lists.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(i64)]
        L.spc_kmap_nnz.argtypes = [vp, ctypes.POINTER(i64)]
        L.spc_kmap_search_info.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.spc_search_count.restype = i64
        L.spc_resident_count.restype = i64
        L.spc_kmap_export_triples.argtypes = [vp, i32, vp, i64, ctypes.POINTER(i64)]
        L.spc_kmap_set_size_hint.argtypes = [vp, i64]
        L.spc_kmap_destroy.argtypes = [vp]
        L.spc_kmap_destroy.restype = None
        L.spc_conv_forward.argtypes = [vp, vp, i64, vp, vp, i64, i32, i32, i32, i32, i32, vp]
        L.spc_conv_forward_hybrid.argtypes = [vp, vp, i64, vp, vp, i64, i32, i32, i32, i32, i32, vp]
        L.spc_conv_prepare_weights.argtypes = [vp, i32, i32, i32, i32, vp, vp]
        L.spc_conv_tune_threshold.argtypes = [vp, vp, i64, vp, vp, vp, i64, i32, i32, i32, i32, i32, ctypes.c_float,
                                              ctypes.POINTER(ctypes.c_float), i32, ctypes.POINTER(i32), ctypes.POINTER(i32), vp]
        L.spc_permute_rows.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp]
        f32, ad, ar = ctypes.c_float, ctypes.POINTER(AttnDesc), ctypes.POINTER(AttnRows)
        L.spc_layer_norm_forward.argtypes = [vp, i64, vp, i64, vp, vp, f32, vp, i64, vp, i64, vp, vp, i64, i32, i32, vp]
        L.spc_layer_norm_backward.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, i64, i32, i32, vp]
        L.spc_rms_norm_forward.argtypes = [vp, i64, vp, i64, vp, f32, vp, i64, vp, i64, vp, i64, i32, i32, vp]
        L.spc_rms_norm_quantize.argtypes = [vp, i64, vp, i64, vp, f32, vp, i64, vp, vp, i64, vp, i64, i32, i32, vp]
        L.spc_quantize_rows.argtypes = [vp, i64, vp, i64, vp, i64, i32, i32, vp]
        L.spc_rms_norm_backward.argtypes = [vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, i64, i32, i32, vp]
        L.spc_linear_f8.argtypes = [vp, i64, vp, vp, i64, vp, vp, i64, i64, i32, i32, i32, vp]
        L.spc_causal_conv_forward.argtypes = [vp, i64, vp, vp, i32, i32, vp, i32, vp, vp, i64, vp, i64, i32, i32, vp]
        L.spc_causal_conv_backward.argtypes = [vp, i64, vp, i64, vp, vp, i32, i32, vp, i32, vp, vp, vp, i64, vp, vp, vp, i64, i32, i32, vp]
        L.spc_causal_conv_step.argtypes = [vp, i64, vp, vp, i32, i32, vp, vp, i64, i64, i32, i32, vp]
        sd = ctypes.POINTER(ScanDesc)
        L.spc_selective_scan_forward.argtypes = [sd, vp, i64, vp, i64, vp, ar, ar, vp, vp, i64, vp, vp, vp, vp, i64, vp, vp]
        L.spc_selective_scan_backward.argtypes = [sd, vp, i64, vp, i64, vp, i64, vp, ar, ar, vp, vp, i64, vp, vp, vp, vp, vp, i64, vp, i64, vp, ar, ar, vp, vp,
                                                  i64, vp, vp, vp]
        L.spc_selective_scan_step.argtypes = [sd, vp, i64, vp, i64, vp, ar, ar, vp, vp, i64, vp, vp, vp, i64, vp]
        L.spc_linear_attention_forward.argtypes = [ad, ar, ar, ar, vp, vp, vp, ar, vp, vp]
        L.spc_linear_attention_backward.argtypes = [ad, ar, ar, ar, ar, vp, vp, vp, vp, ar, ar, ar, vp, vp]
        L.spc_linear_attention_step.argtypes = [ad, ar, ar, ar, vp, vp, ar, vp]
        L.spc_batch_offsets.argtypes = [vp, i64, ctypes.POINTER(PackDesc), i32, vp, vp]
        L.spc_probe_copy.argtypes = [vp, vp, i64, vp]
        L.spc_probe_mfma.argtypes = [i32, vp, ctypes.POINTER(ctypes.c_double), vp]
        L.spc_last_error.restype = ctypes.c_char_p
        L.spc_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != OK:
        raise SpcError(rc, lib().spc_last_error().decode())


def current_raw_stream() -> int:
    """Handle of torch's current stream (a torch.cuda.Stream object costs 2.8 us per call, the handle alone 0.1)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _stream(stream=None) -> int:
    if stream is None:
        return current_raw_stream()
    return int(stream) if isinstance(stream, int) or not hasattr(stream, "cuda_stream") else int(stream.cuda_stream)


def _dev_ptr(t: torch.Tensor) -> int:
    assert t.is_cuda and t.is_contiguous()
    return t.data_ptr()


_TORCH_DTYPE = {torch.float16: DTYPE_F16, torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}


def spc_version() -> str:
    return lib().spc_version().decode()


def spc_pack_desc_fit(lo, hi, n_batch: int = 1, max_stride: int = 1, max_reach: int = 1, key_bits: int = 0) -> PackDesc:
    d = PackDesc()
    a = (ctypes.c_int32 * 3)(*[int(v) for v in lo])
    b = (ctypes.c_int32 * 3)(*[int(v) for v in hi])
    _check(lib().spc_pack_desc_fit(a, b, n_batch, max_stride, max_reach, key_bits, ctypes.byref(d)))
    return d


def spc_pack_workspace_bytes(n: int, desc: PackDesc) -> int:
    need = ctypes.c_size_t(0)
    _check(lib().spc_pack_coords(None, n, ctypes.byref(desc), None, None, None, ctypes.byref(need), 0, None))
    return int(need.value)


def spc_pack_coords(coords: torch.Tensor, desc: PackDesc, want_perm: bool = True, flags: int = 0, stream=None,
                    workspace: torch.Tensor | None = None, keys_out: torch.Tensor | None = None,
                    perm_out: torch.Tensor | None = None):
    """coords: int32 [N,4] device tensor (b,x,y,z).  Returns (keys, perm): sorted packed keys
    (int32/int64 tensors holding the unsigned bit patterns) and the permutation (or None)."""
    # (every attribute of a tensor costs about 0.1 us of host time, and a call reads some twenty: each is read once)
    shape = coords.shape
    assert coords.dtype == torch.int32 and len(shape) == 2 and shape[1] == 4
    n = shape[0]
    if workspace is None:
        workspace = torch.empty(spc_pack_workspace_bytes(n, desc), dtype=torch.uint8, device=coords.device)
    kdt = torch.int32 if desc.key_bits == 32 else torch.int64
    keys = keys_out if keys_out is not None else torch.empty(n, dtype=kdt, device=coords.device)
    assert keys.dtype == kdt and keys.numel() == n
    perm = None
    if want_perm:
        perm = perm_out if perm_out is not None else torch.empty(n, dtype=torch.int32, device=coords.device)
        assert perm.dtype == torch.int32 and perm.numel() == n
    size = ctypes.c_size_t(workspace.numel())
    rc = lib().spc_pack_coords(_dev_ptr(coords), n, ctypes.byref(desc), _dev_ptr(keys), _dev_ptr(perm) if want_perm else None,
                               _dev_ptr(workspace), ctypes.byref(size), flags, current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return keys, perm


NOALLOC_MAX_N = 262144


def spc_pack_coords_noalloc(coords: torch.Tensor, desc: PackDesc, keys_out: torch.Tensor, perm_out: torch.Tensor | None,
                            flags: int = 0, stream=None) -> None:
    """spc_pack_coords on the library's static scratch buffer: the caller passes inputs and outputs only."""
    assert coords.dtype == torch.int32 and coords.dim() == 2 and coords.shape[1] == 4
    n = coords.shape[0]
    assert keys_out.dtype == (torch.int32 if desc.key_bits == 32 else torch.int64) and keys_out.numel() == n
    assert perm_out is None or (perm_out.dtype == torch.int32 and perm_out.numel() == n)
    _check(lib().spc_pack_coords_noalloc(_dev_ptr(coords), n, ctypes.byref(desc), _dev_ptr(keys_out),
                                         _dev_ptr(perm_out) if perm_out is not None else None, flags, _stream(stream)))


class KMap:
    """Owner of one spc_kmap handle (keeps the key tensor it points into alive)."""

    def __init__(self, handle: int, keep=(), desc: PackDesc | None = None):
        self.handle = ctypes.c_void_p(handle)
        self._keep = keep
        self._kvol = None
        self.desc = desc

    def destroy(self):
        if self.handle:
            lib().spc_kmap_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            if self.handle:
                self.destroy()
        except Exception:
            pass

    @property
    def n_in(self) -> int:
        v = lib().spc_kmap_n_in(self.handle)
        if v < 0:
            _check(int(v))
        return int(v)

    @property
    def n_out(self) -> int:
        v = lib().spc_kmap_n_out(self.handle)
        if v < 0:
            _check(int(v))
        return int(v)

    def set_size_hint(self, n_out_hint: int) -> None:
        _check(lib().spc_kmap_set_size_hint(self.handle, int(n_out_hint)))

    @property
    def kvol(self) -> int:
        if self._kvol is None:
            self._kvol = int(lib().spc_kmap_kvol(self.handle))
        return self._kvol

    def nnz(self):
        import numpy as np
        out = np.zeros(self.kvol, dtype=np.int64)
        _check(lib().spc_kmap_nnz(self.handle, out.ctypes.data_as(ctypes.POINTER(ctypes.c_int64))))
        return out

    def export_triples(self, which: int = LAYOUT_OS):
        import numpy as np
        nnz = ctypes.c_int64(0)
        _check(lib().spc_kmap_export_triples(self.handle, which, None, 0, ctypes.byref(nnz)))
        t = np.empty((nnz.value, 3), dtype=np.int32)
        _check(lib().spc_kmap_export_triples(self.handle, which, t.ctypes.data_as(ctypes.c_void_p), nnz.value,
                                             ctypes.byref(nnz)))
        return t

    def out_keys(self):
        """Host copy of the layer's sorted output keys (as uint64)."""
        import numpy as np
        n = self.n_out
        a = np.empty(n, dtype=np.uint32 if self.desc.key_bits == 32 else np.uint64)
        _check(lib().spc_kmap_copy_out_keys(self.handle, a.ctypes.data_as(ctypes.c_void_p), n))
        return a.astype(np.uint64)


def spc_search_count() -> int:
    """Kernel-map searches enqueued by this process so far."""
    return int(lib().spc_search_count())


def spc_resident_count() -> int:
    """Feature calls enqueued by this process so far that took the kernel with resident weights."""
    return int(lib().spc_resident_count())


def spc_kmap_search_info(kmap: KMap):
    """(rows per search tile, input keys the tile's windows may occupy in LDS)."""
    t, w = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().spc_kmap_search_info(kmap.handle, ctypes.byref(t), ctypes.byref(w)))
    return int(t.value), int(w.value)


_layer_desc_of: dict = {}  # layer descriptors in C form (read only) by their values, the first few hundred


def spc_build_kmap(in_keys: torch.Tensor, desc: PackDesc, K: int, in_stride: int = 1, layer_stride: int = 1,
                   transposed: int = 0, layout: int = LAYOUT_BOTH, stream=None, in_perm: torch.Tensor | None = None) -> KMap:
    """in_perm: the permutation returned by spc_pack_coords; the map then addresses the caller's unsorted
    feature rows (spc_build_kmap_perm)."""
    key = (K, in_stride, layer_stride, transposed, layout)
    l = _layer_desc_of.get(key)
    if l is None:
        l = LayerDesc(*key)
        if len(_layer_desc_of) < 256:
            _layer_desc_of[key] = l
    h = ctypes.c_void_p()
    n, raw = in_keys.shape[0], current_raw_stream() if stream is None else _stream(stream)
    if in_perm is None:
        rc = lib().spc_build_kmap(_dev_ptr(in_keys), n, ctypes.byref(desc), ctypes.byref(l), ctypes.byref(h), raw)
    else:
        assert in_perm.dtype == torch.int32 and in_perm.shape[0] == n
        rc = lib().spc_build_kmap_perm(_dev_ptr(in_keys), n, _dev_ptr(in_perm), ctypes.byref(desc), ctypes.byref(l), ctypes.byref(h), raw)
    if rc:
        _check(rc)
    return KMap(h.value, keep=(in_keys, in_perm), desc=desc)


def layer_descs(layers):
    """The C form of a sequence of (K, in_stride, layer_stride, transposed, layout)."""
    return (LayerDesc * len(layers))(*[LayerDesc(*[int(v) for v in l]) for l in layers])


def spc_build_kmaps_network(v0_keys: torch.Tensor, desc: PackDesc, layers, streams=None, flags: int = 0):
    """layers: sequence of (K, in_stride, layer_stride, transposed, layout), or what layer_descs() made of one.  Returns
    one KMap per layer (layers with equal (K, in_stride, layer_stride, transposed) share the underlying map)."""
    n = len(layers)
    arr = layers if isinstance(layers, ctypes.Array) else layer_descs(layers)
    out = (ctypes.c_void_p * n)()
    if streams is None:
        streams = [torch.cuda.current_stream()]
    sarr = (ctypes.c_void_p * len(streams))(*[_stream(s) for s in streams])
    _check(lib().spc_build_kmaps_network(_dev_ptr(v0_keys), v0_keys.shape[0], ctypes.byref(desc), arr, n, out, sarr,
                                         len(streams), flags))
    return [KMap(out[i], keep=(v0_keys,), desc=desc) for i in range(n)]


def spc_conv_forward(kmap: KMap, feats_in: torch.Tensor, weights: torch.Tensor, dataflow: int = DATAFLOW_OS,
                     flags: int = 0, out: torch.Tensor | None = None, n_out: int | None = None, stream=None,
                     hybrid_t: int | None = None) -> torch.Tensor:
    """feats_in [n_in, cin] (row pitch = stride(0)), weights [K^3, cin, cout] contiguous.  ``out`` may be a
    column slice of a wider buffer (row pitch = stride(0)); it is allocated when None.  hybrid_t: threshold of the
    hybrid dual dataflow (spc_conv_forward_hybrid); `dataflow` is ignored then."""
    assert feats_in.is_cuda and weights.is_cuda and weights.is_contiguous()
    fs, ws, fst, dtype = feats_in.shape, weights.shape, feats_in.stride(), feats_in.dtype
    assert len(fs) == 2 and fst[1] == 1 and len(ws) == 3
    code = _TORCH_DTYPE.get(dtype)
    assert dtype == weights.dtype and code is not None
    kvol, wcin, cout = ws
    cin = fs[1]
    # (prepacked weights hold their input channels padded to a multiple of 16)
    assert wcin == ((cin + 15) // 16 * 16 if flags & CONV_PACKED_WEIGHTS else cin) and kvol == kmap.kvol
    if out is None:
        out = torch.empty((n_out if n_out is not None else kmap.n_out, cout), dtype=dtype, device=feats_in.device)
    oshape, ost = out.shape, out.stride()
    assert len(oshape) == 2 and ost[1] == 1 and oshape[1] == cout and out.dtype == dtype
    raw = current_raw_stream() if stream is None else _stream(stream)
    if hybrid_t is not None:
        rc = lib().spc_conv_forward_hybrid(kmap.handle, feats_in.data_ptr(), fst[0], weights.data_ptr(), out.data_ptr(), ost[0], cin,
                                           cout, code, int(hybrid_t), flags, raw)
    else:
        rc = lib().spc_conv_forward(kmap.handle, feats_in.data_ptr(), fst[0], weights.data_ptr(), out.data_ptr(), ost[0], cin, cout,
                                    code, dataflow, flags, raw)
    if rc:
        _check(rc)
    return out


def spc_conv_tune_threshold(kmap: KMap, feats_in: torch.Tensor, weights: torch.Tensor, packed: torch.Tensor | None = None,
                            flags: int = 0, reps: int = 5, ws_build_us: float = 0.0, out: torch.Tensor | None = None,
                            stream=None):
    """One-time tuning of a layer's hybrid threshold (spc_conv_tune_threshold).  Returns (best t, [microseconds for
    t = 0 .. L1max + 1], output computed with the best t)."""
    assert feats_in.is_cuda and weights.is_cuda and weights.is_contiguous() and weights.dim() == 3
    assert feats_in.dim() == 2 and feats_in.stride(1) == 1 and feats_in.dtype == weights.dtype and feats_in.dtype in _TORCH_DTYPE
    cin, cout = weights.shape[1], weights.shape[2]
    assert feats_in.shape[1] == cin and weights.shape[0] == kmap.kvol
    assert packed is None or (packed.is_cuda and packed.is_contiguous() and packed.dtype == weights.dtype
                              and packed.numel() == weights.shape[0] * ((weights.shape[1] + 15) // 16 * 16) * weights.shape[2])
    if out is None:
        out = torch.empty((kmap.n_out, cout), dtype=feats_in.dtype, device=feats_in.device)
    assert out.dim() == 2 and out.stride(1) == 1 and out.shape[1] == cout and out.dtype == feats_in.dtype
    cap = 64
    us = (ctypes.c_float * cap)()
    n_t, best = ctypes.c_int32(0), ctypes.c_int32(-1)
    _check(lib().spc_conv_tune_threshold(kmap.handle, feats_in.data_ptr(), feats_in.stride(0), weights.data_ptr(),
                                         packed.data_ptr() if packed is not None else None, out.data_ptr(), out.stride(0), cin,
                                         cout, _TORCH_DTYPE[feats_in.dtype], flags, int(reps), float(ws_build_us), us, cap,
                                         ctypes.byref(n_t), ctypes.byref(best), _stream(stream)))
    return int(best.value), [float(us[i]) for i in range(n_t.value)], out


def spc_conv_prepare_weights(weights: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """weights [K^3, cin, cout] fp16/bf16 -> the MFMA operand layout expected with CONV_PACKED_WEIGHTS."""
    assert weights.is_cuda and weights.is_contiguous() and weights.dim() == 3 and weights.dtype in _TORCH_DTYPE
    cin16 = (weights.shape[1] + 15) // 16 * 16  # input channels are padded with zeros to a multiple of 16
    if out is None:
        out = torch.empty((weights.shape[0], cin16, weights.shape[2]), dtype=weights.dtype, device=weights.device)
    assert out.is_contiguous() and out.dtype == weights.dtype and out.numel() == weights.shape[0] * cin16 * weights.shape[2]
    _check(lib().spc_conv_prepare_weights(weights.data_ptr(), weights.shape[0], weights.shape[1], weights.shape[2],
                                          _TORCH_DTYPE[weights.dtype], out.data_ptr(), _stream(stream)))
    return out


def spc_permute_rows(src: torch.Tensor, perm: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """out[r] = src[perm[r]] (feature rows into sorted-voxel order)."""
    assert src.is_cuda and src.dim() == 2 and src.stride(1) == 1 and perm.dtype == torch.int32
    if out is None:
        out = torch.empty((perm.shape[0], src.shape[1]), dtype=src.dtype, device=src.device)
    es = src.element_size()
    _check(lib().spc_permute_rows(src.data_ptr(), src.stride(0) * es, perm.data_ptr(), perm.shape[0], src.shape[1] * es,
                                  out.data_ptr(), out.stride(0) * es, _stream(stream)))
    return out


def _norm_rows(t: torch.Tensor, like: torch.Tensor) -> int:
    """Row pitch of a matrix of like's shape and type on its device."""
    st = t.stride()
    assert t.is_cuda and t.device == like.device and t.dtype == like.dtype and t.shape == like.shape
    assert len(st) == 2 and (st[1] == 1 or t.shape[1] <= 1)
    # (the pitch of a matrix of one row may be anything)
    return st[0] if t.shape[0] > 1 else max(st[0], t.shape[1])


def _f32(t: torch.Tensor | None, shape, device) -> int | None:
    """Pointer of an optional contiguous fp32 tensor of this shape."""
    if t is None:
        return None
    assert t.dtype == torch.float32 and t.shape == shape and t.is_contiguous() and t.device == device
    return t.data_ptr()


def spc_layer_norm_forward(x: torch.Tensor, gamma: torch.Tensor | None = None, beta: torch.Tensor | None = None, eps: float = 1e-5,
                           residual: torch.Tensor | None = None, out: torch.Tensor | None = None, sum_out: torch.Tensor | None = None,
                           want_stats: bool = False, stream=None):
    """Layer norm of the rows of x [n, c] (+ residual); gamma, beta [c] fp32.  Row pitches = stride(0).  Returns (y, sum, mean, rstd): sum is
    None without a residual, mean and rstd [n] fp32 are None without want_stats."""
    (n, c), dev, dtype, ld = x.shape, x.device, x.dtype, _norm_rows(x, x)
    code = _TORCH_DTYPE.get(dtype)
    assert code is not None
    # (tensors made here need no checks; each costs a call of some 10 us about half of one)
    y, ld_y, total, ld_s = out, c, None, c
    if out is None:
        y = torch.empty(n, c, dtype=dtype, device=dev)
    else:
        ld_y = _norm_rows(out, x)
    if residual is None:
        assert sum_out is None
    elif sum_out is None:
        total = torch.empty(n, c, dtype=dtype, device=dev)
    else:
        total, ld_s = sum_out, _norm_rows(sum_out, x)
    mean = rstd = None
    if want_stats:
        mean, rstd = torch.empty(n, dtype=torch.float32, device=dev), torch.empty(n, dtype=torch.float32, device=dev)
    rc = lib().spc_layer_norm_forward(x.data_ptr(), ld, residual.data_ptr() if residual is not None else None,
                                      _norm_rows(residual, x) if residual is not None else 0, _f32(gamma, (c,), dev), _f32(beta, (c,), dev),
                                      eps, y.data_ptr(), ld_y, total.data_ptr() if total is not None else None, ld_s,
                                      mean.data_ptr() if want_stats else None, rstd.data_ptr() if want_stats else None, n, c, code,
                                      current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return y, total, mean, rstd


def spc_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, gamma: torch.Tensor | None = None,
                            dsum: torch.Tensor | None = None, out: torch.Tensor | None = None, want_params: bool = True, stream=None):
    """Gradients of spc_layer_norm_forward; x is its x, or its sum where there was a residual, dsum [n, c] a gradient that reaches that sum past
    the norm.  Returns (dx, dgamma, dbeta), the last two [c] fp32, or None without want_params."""
    (n, c), dev, ld = x.shape, x.device, _norm_rows(x, x)
    code = _TORCH_DTYPE.get(x.dtype)
    assert code is not None
    dx, ld_dx = out, c
    if out is None:
        dx = torch.empty(n, c, dtype=x.dtype, device=dev)
    else:
        ld_dx = _norm_rows(out, x)
    dgamma = dbeta = None
    if want_params:
        dgamma, dbeta = torch.empty(c, dtype=torch.float32, device=dev), torch.empty(c, dtype=torch.float32, device=dev)
    rc = lib().spc_layer_norm_backward(dy.data_ptr(), _norm_rows(dy, x), x.data_ptr(), ld, _f32(mean, (n,), dev),
                                       _f32(rstd, (n,), dev), _f32(gamma, (c,), dev), dsum.data_ptr() if dsum is not None else None,
                                       _norm_rows(dsum, x) if dsum is not None else 0, dx.data_ptr(), ld_dx,
                                       dgamma.data_ptr() if want_params else None, dbeta.data_ptr() if want_params else None, n, c, code,
                                       current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return dx, dgamma, dbeta


def _heads(t: torch.Tensor, n: int, heads: int, width: int, dtype, dev) -> AttnRows:
    row, head, channel = t.stride()
    assert t.dtype == dtype and t.device == dev and t.shape == (n, heads, width) and (channel == 1 or width == 1)
    return AttnRows(t.data_ptr(), row, head)


def _attention(q, k, v, log_decay, offsets, scale):
    """What the calls share: (descriptor, q, k, v in C form, log_decay's and offsets' addresses)."""
    n, heads, dk = q.shape
    _, kv, dv = v.shape
    dev, dtype, n_scenes, at = q.device, q.dtype, 1, None
    code = _TORCH_DTYPE.get(dtype)
    assert q.is_cuda and code is not None
    if offsets is not None:
        n_scenes, at = offsets.shape[0] - 1, offsets.data_ptr()
        assert offsets.dtype == torch.int32 and offsets.dim() == 1 and offsets.is_contiguous() and offsets.device == dev
    d = AttnDesc(code, n_scenes, n, heads, kv, dk, dv, dk ** -0.5 if scale is None else scale)
    return (d, _heads(q, n, heads, dk, dtype, dev), _heads(k, n, kv, dk, dtype, dev), _heads(v, n, kv, dv, dtype, dev),
            _f32(log_decay, (heads,), dev), at)


def spc_linear_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor, offsets: torch.Tensor | None = None,
                                 scale: float | None = None, initial_state: torch.Tensor | None = None, want_state: bool = False,
                                 out: torch.Tensor | None = None, state_out: torch.Tensor | None = None, stream=None):
    """q [n, heads, dk], k [n, kv_heads, dk], v [n, kv_heads, dv] (any row and head pitch, e.g. column ranges of one projection's output);
    log_decay [heads] fp32, <= 0; offsets [scenes + 1] int32 (spc_batch_offsets), None: one scene; scale None: dk ** -0.5; states
    [scenes, heads, dk, dv] fp32.  Returns (out [n, heads, dv], state behind every scene's last row, or None)."""
    d, rq, rk, rv, g, at = _attention(q, k, v, log_decay, offsets, scale)
    n, heads, dev = d.n_rows, d.heads, q.device
    shape = (d.n_scenes, heads, d.dk, d.dv)
    ro = None if out is None else _heads(out, n, heads, d.dv, q.dtype, dev)
    if out is None:
        out = torch.empty(n, heads, d.dv, dtype=q.dtype, device=dev)
        ro = AttnRows(out.data_ptr(), heads * d.dv, d.dv)
    if state_out is None and want_state:
        state_out = torch.empty(shape, dtype=torch.float32, device=dev)
    rc = lib().spc_linear_attention_forward(d, rq, rk, rv, g, at, _f32(initial_state, shape, dev), ro, _f32(state_out, shape, dev),
                                            current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return out, state_out


def spc_linear_attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor,
                                  offsets: torch.Tensor | None = None, scale: float | None = None, initial_state: torch.Tensor | None = None,
                                  dstate: torch.Tensor | None = None, want_dinitial: bool = False, out=None, stream=None):
    """Gradients of spc_linear_attention_forward; dstate: gradient of the state it returned.  out: (dq, dk, dv) to write to.  Returns
    (dq, dk, dv, gradient of initial_state or None)."""
    d, rq, rk, rv, g, at = _attention(q, k, v, log_decay, offsets, scale)
    n, heads, kv, dev = d.n_rows, d.heads, d.kv_heads, q.device
    shape = (d.n_scenes, heads, d.dk, d.dv)
    if out is None:
        out = tuple(torch.empty(*s, dtype=q.dtype, device=dev) for s in ((n, heads, d.dk), (n, kv, d.dk), (n, kv, d.dv)))
    dinitial = torch.empty(shape, dtype=torch.float32, device=dev) if want_dinitial else None
    rc = lib().spc_linear_attention_backward(d, _heads(dout, n, heads, d.dv, q.dtype, dev), rq, rk, rv, g, at, _f32(initial_state, shape, dev),
                                             _f32(dstate, shape, dev), _heads(out[0], n, heads, d.dk, q.dtype, dev), _heads(out[1], n, kv, d.dk, q.dtype, dev),
                                             _heads(out[2], n, kv, d.dv, q.dtype, dev), _f32(dinitial, shape, dev),
                                             current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return (*out, dinitial)


def spc_linear_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor, state: torch.Tensor,
                              scale: float | None = None, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """One more row for every stream: q [streams, heads, dk] and so on; state [streams, heads, dk, dv] fp32 is updated in place."""
    d, rq, rk, rv, g, _ = _attention(q, k, v, log_decay, None, scale)
    n, heads, dk, dv, dev = d.n_rows, d.heads, d.dk, d.dv, q.device
    ro = None if out is None else _heads(out, n, heads, dv, q.dtype, dev)
    if out is None:
        out = torch.empty(n, heads, dv, dtype=q.dtype, device=dev)
        ro = AttnRows(out.data_ptr(), heads * dv, dv)
    rc = lib().spc_linear_attention_step(d, rq, rk, rv, g, _f32(state, (n, heads, dk, dv), dev), ro, current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return out


def _opt_rows(t: torch.Tensor | None, like: torch.Tensor):
    """(address, row pitch) of an optional matrix of like's shape and type."""
    return (None, 0) if t is None else (t.data_ptr(), _norm_rows(t, like))


def _code(t: torch.Tensor) -> int:
    code = _TORCH_DTYPE.get(t.dtype)
    assert code is not None
    return code


def spc_rms_norm_forward(x: torch.Tensor, gamma: torch.Tensor | None = None, eps: float = 1e-5, residual: torch.Tensor | None = None,
                         out: torch.Tensor | None = None, sum_out: torch.Tensor | None = None, want_stats: bool = False, stream=None):
    """Root-mean-square norm of the rows of x [n, c] (+ residual); gamma [c] fp32.  Returns (y, sum, rstd): sum is None without a residual,
    rstd [n] fp32 None without want_stats."""
    (n, c), dev, code, ld = x.shape, x.device, _code(x), _norm_rows(x, x)
    assert residual is not None or sum_out is None
    r, ld_r = _opt_rows(residual, x)
    y = torch.empty(n, c, dtype=x.dtype, device=dev) if out is None else out
    total = torch.empty(n, c, dtype=x.dtype, device=dev) if residual is not None and sum_out is None else sum_out
    rstd = torch.empty(n, dtype=torch.float32, device=dev) if want_stats else None
    rc = lib().spc_rms_norm_forward(x.data_ptr(), ld, r, ld_r, _f32(gamma, (c,), dev), eps, y.data_ptr(), c if out is None else _norm_rows(out, x),
                                    None if total is None else total.data_ptr(), c if sum_out is None else _norm_rows(sum_out, x),
                                    rstd.data_ptr() if want_stats else None, n, c, code, current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return y, total, rstd


def _bytes(q: torch.Tensor, n: int, c: int, dev) -> int:
    """Row pitch of a matrix of e4m3 values."""
    st = q.stride()
    assert q.dtype == torch.float8_e4m3fn and q.shape == (n, c) and q.device == dev and q.is_cuda and (st[1] == 1 or c <= 1)
    return st[0] if n > 1 else max(st[0], c)


def spc_rms_norm_quantize(x: torch.Tensor, gamma: torch.Tensor | None = None, eps: float = 1e-5, residual: torch.Tensor | None = None,
                          out: torch.Tensor | None = None, scale_out: torch.Tensor | None = None, sum_out: torch.Tensor | None = None,
                          want_stats: bool = False, stream=None):
    """The same norm with its output in 8 bits: returns (q [n, c] float8_e4m3fn, scale [n] fp32, sum, rstd), y being q times its row's scale."""
    (n, c), dev, code, ld = x.shape, x.device, _code(x), _norm_rows(x, x)
    assert residual is not None or sum_out is None
    r, ld_r = _opt_rows(residual, x)
    q = torch.empty(n, c, dtype=torch.float8_e4m3fn, device=dev) if out is None else out
    scale = torch.empty(n, dtype=torch.float32, device=dev) if scale_out is None else scale_out
    total = torch.empty(n, c, dtype=x.dtype, device=dev) if residual is not None and sum_out is None else sum_out
    rstd = torch.empty(n, dtype=torch.float32, device=dev) if want_stats else None
    rc = lib().spc_rms_norm_quantize(x.data_ptr(), ld, r, ld_r, _f32(gamma, (c,), dev), eps, q.data_ptr(), c if out is None else _bytes(out, n, c, dev),
                                     _f32(scale, (n,), dev), None if total is None else total.data_ptr(),
                                     c if sum_out is None else _norm_rows(sum_out, x), rstd.data_ptr() if want_stats else None, n, c, code,
                                     current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return q, scale, total, rstd


def spc_quantize_rows(x: torch.Tensor, out: torch.Tensor | None = None, scale_out: torch.Tensor | None = None, stream=None):
    """Rows of x [n, c] in 8 bits: (q [n, c] float8_e4m3fn, scale [n] fp32).  Weights for spc_linear_f8 are quantised as [cout, cin]."""
    (n, c), dev, code, ld = x.shape, x.device, _code(x), _norm_rows(x, x)
    q = torch.empty(n, c, dtype=torch.float8_e4m3fn, device=dev) if out is None else out
    scale = torch.empty(n, dtype=torch.float32, device=dev) if scale_out is None else scale_out
    _check(lib().spc_quantize_rows(x.data_ptr(), ld, q.data_ptr(), _bytes(q, n, c, dev), _f32(scale, (n,), dev), n, c, code,
                                   current_raw_stream() if stream is None else _stream(stream)))
    return q, scale


def spc_rms_norm_backward(dy: torch.Tensor, x: torch.Tensor, rstd: torch.Tensor, gamma: torch.Tensor | None = None, dsum: torch.Tensor | None = None,
                          out: torch.Tensor | None = None, want_params: bool = True, stream=None):
    """Gradients of spc_rms_norm_forward; x is its x, or its sum where there was a residual, dsum a gradient that reaches that sum past the
    norm.  Returns (dx, dgamma), the latter [c] fp32, or None without want_params."""
    (n, c), dev, code, ld = x.shape, x.device, _code(x), _norm_rows(x, x)
    e, ld_e = _opt_rows(dsum, x)
    dx = torch.empty(n, c, dtype=x.dtype, device=dev) if out is None else out
    dgamma = torch.empty(c, dtype=torch.float32, device=dev) if want_params else None
    rc = lib().spc_rms_norm_backward(dy.data_ptr(), _norm_rows(dy, x), x.data_ptr(), ld, _f32(rstd, (n,), dev), _f32(gamma, (c,), dev), e, ld_e,
                                     dx.data_ptr(), c if out is None else _norm_rows(out, x), dgamma.data_ptr() if want_params else None, n, c, code,
                                     current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return dx, dgamma


def spc_linear_f8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, dtype: torch.dtype = torch.bfloat16,
                  out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """1x1x1 layer in 8 bits: x [n, cin] and w [cout, cin] float8_e4m3fn with a scale for each row (spc_rms_norm_quantize, spc_quantize_rows).
    Returns [n, cout] of `dtype` (or of out's)."""
    (n, c), (m, _), dev = x.shape, w.shape, x.device
    if out is None:
        out = torch.empty(n, m, dtype=dtype, device=dev)
    assert out.shape == (n, m) and out.device == dev
    rc = lib().spc_linear_f8(x.data_ptr(), _bytes(x, n, c, dev), _f32(x_scale, (n,), dev), w.data_ptr(), _bytes(w, m, c, dev), _f32(w_scale, (m,), dev),
                             out.data_ptr(), _norm_rows(out, out), n, c, m, _code(out), current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return out


def _scenes_of(offsets: torch.Tensor | None, dev):
    """(number of scenes, address of their offsets)."""
    if offsets is None:
        return 1, None
    assert offsets.dtype == torch.int32 and offsets.dim() == 1 and offsets.is_contiguous() and offsets.device == dev
    return offsets.shape[0] - 1, offsets.data_ptr()


def _past(t: torch.Tensor | None, shape, like: torch.Tensor) -> int | None:
    """Address of optional contiguous rows in front of scenes or streams, of like's type."""
    if t is None:
        return None
    assert t.shape == shape and t.dtype == like.dtype and t.device == like.device and t.is_contiguous()
    return t.data_ptr()


def spc_causal_conv_forward(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                            silu: bool = True, initial_rows: torch.Tensor | None = None, want_rows: bool = False, out: torch.Tensor | None = None,
                            rows_out: torch.Tensor | None = None, stream=None):
    """Short causal convolution of every channel of x [n, c] along the rows of its scene, through x / (1 + exp(-x)) with silu; weight [c, width] (the
    row itself last) and bias [c] fp32; offsets [scenes + 1] int32 (spc_batch_offsets), None: one scene.  initial_rows [scenes, width - 1, c] of x's
    type: the rows in front of each scene.  Returns (y [n, c], every scene's last width - 1 rows or None)."""
    (n, c), dev, code, ld = x.shape, x.device, _code(x), _norm_rows(x, x)
    width, (scenes, at) = weight.shape[1], _scenes_of(offsets, dev)
    shape = (scenes, width - 1, c)
    y = torch.empty(n, c, dtype=x.dtype, device=dev) if out is None else out
    if rows_out is None and want_rows:
        rows_out = torch.empty(shape, dtype=x.dtype, device=dev)
    rc = lib().spc_causal_conv_forward(x.data_ptr(), ld, _f32(weight, (c, width), dev), _f32(bias, (c,), dev), width, bool(silu), at, scenes,
                                       _past(initial_rows, shape, x), y.data_ptr(), c if out is None else _norm_rows(out, x),
                                       _past(rows_out, shape, x), n, c, code, current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return y, rows_out


def spc_causal_conv_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                             silu: bool = True, initial_rows: torch.Tensor | None = None, drows: torch.Tensor | None = None, want_params: bool = True,
                             want_dinitial: bool = False, out: torch.Tensor | None = None, stream=None):
    """Gradients of spc_causal_conv_forward; drows: gradient of the rows it returned.  Returns (dx, dweight, dbias, gradient of initial_rows), the
    second and third None without want_params, the last without want_dinitial."""
    (n, c), dev, code, ld = x.shape, x.device, _code(x), _norm_rows(x, x)
    width, (scenes, at) = weight.shape[1], _scenes_of(offsets, dev)
    shape = (scenes, width - 1, c)
    dx = torch.empty(n, c, dtype=x.dtype, device=dev) if out is None else out
    dweight = torch.empty(c, width, dtype=torch.float32, device=dev) if want_params else None
    dbias = torch.empty(c, dtype=torch.float32, device=dev) if want_params else None
    dinitial = torch.empty(shape, dtype=x.dtype, device=dev) if want_dinitial else None
    rc = lib().spc_causal_conv_backward(dy.data_ptr(), _norm_rows(dy, x), x.data_ptr(), ld, _f32(weight, (c, width), dev), _f32(bias, (c,), dev), width,
                                        bool(silu), at, scenes, _past(initial_rows, shape, x), _past(drows, shape, x), dx.data_ptr(),
                                        c if out is None else _norm_rows(out, x), dweight.data_ptr() if want_params else None,
                                        dbias.data_ptr() if want_params else None, dinitial.data_ptr() if want_dinitial else None, n, c, code,
                                        current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return dx, dweight, dbias, dinitial


def spc_causal_conv_step(x: torch.Tensor, weight: torch.Tensor, rows: torch.Tensor, bias: torch.Tensor | None = None, silu: bool = True,
                         out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """One more row x [streams, c] of every stream; rows [streams, width - 1, c], the streams' last ones, are updated in place."""
    (n, c), dev, code, ld = x.shape, x.device, _code(x), _norm_rows(x, x)
    width = weight.shape[1]
    y = torch.empty(n, c, dtype=x.dtype, device=dev) if out is None else out
    rc = lib().spc_causal_conv_step(x.data_ptr(), ld, _f32(weight, (c, width), dev), _f32(bias, (c,), dev), width, bool(silu),
                                    _past(rows, (n, width - 1, c), x), y.data_ptr(), c if out is None else _norm_rows(out, x), n, c, code,
                                    current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return y


def _scan(u, dt, A, b, c, skip, gate, dt_bias, offsets, softplus):
    """What the scan's calls share: (descriptor, arguments from u to dt_bias in C form, offsets' address)."""
    n, channels = u.shape
    groups, states = b.shape[1], A.shape[1]
    dev = u.device
    scenes, at = _scenes_of(offsets, dev)
    d = ScanDesc(_code(u), scenes, n, channels, groups, states, bool(softplus))
    z, ld_z = _opt_rows(gate, u)
    return d, (u.data_ptr(), _norm_rows(u, u), dt.data_ptr(), _norm_rows(dt, u), _f32(A, (channels, states), dev), _heads(b, n, groups, states, u.dtype, dev),
               _heads(c, n, groups, states, u.dtype, dev), _f32(skip, (channels,), dev), z, ld_z, _f32(dt_bias, (channels,), dev)), at


def spc_selective_scan_forward(u: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, skip: torch.Tensor | None = None,
                               gate: torch.Tensor | None = None, dt_bias: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                               softplus: bool = True, initial_state: torch.Tensor | None = None, want_state: bool = False,
                               out: torch.Tensor | None = None, state_out: torch.Tensor | None = None, stream=None):
    """Selective scan along every scene's rows: u, dt, gate [n, channels], B, C [n, groups, states] (any row and group pitch, e.g. column ranges of one
    projection's output); A [channels, states], skip and dt_bias [channels] fp32; step sizes dt + dt_bias, through ln(1 + exp) with softplus; offsets
    [scenes + 1] int32 (spc_batch_offsets), None: one scene; states [scenes, channels, states] fp32.  Returns (out [n, channels], state behind
    every scene's last row, or None)."""
    d, args, at = _scan(u, dt, A, B, C, skip, gate, dt_bias, offsets, softplus)
    dev = u.device
    shape = (d.n_scenes, d.channels, d.states)
    y = torch.empty(d.n_rows, d.channels, dtype=u.dtype, device=dev) if out is None else out
    if state_out is None and want_state:
        state_out = torch.empty(shape, dtype=torch.float32, device=dev)
    rc = lib().spc_selective_scan_forward(d, *args, at, _f32(initial_state, shape, dev), y.data_ptr(), d.channels if out is None else _norm_rows(out, u),
                                          _f32(state_out, shape, dev), current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return y, state_out


def spc_selective_scan_backward(dout: torch.Tensor, u: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor,
                                skip: torch.Tensor | None = None, gate: torch.Tensor | None = None, dt_bias: torch.Tensor | None = None,
                                offsets: torch.Tensor | None = None, softplus: bool = True, initial_state: torch.Tensor | None = None,
                                dstate: torch.Tensor | None = None, want_dinitial: bool = False, out=None, stream=None) -> ScanGradients:
    """Gradients of spc_selective_scan_forward; dstate: gradient of the state it returned.  out: (du, ddt, dB, dC, dgate or None) to write to.  Returns
    ScanGradients; skip, gate and dt_bias have none where they were None, initial without want_dinitial."""
    d, args, at = _scan(u, dt, A, B, C, skip, gate, dt_bias, offsets, softplus)
    dev, n, ch = u.device, d.n_rows, d.channels
    shape = (d.n_scenes, ch, d.states)
    if out is None:
        rows = lambda: torch.empty(n, ch, dtype=u.dtype, device=dev)  # noqa: E731
        low = lambda: torch.empty(n, d.groups, d.states, dtype=u.dtype, device=dev)  # noqa: E731
        out = (rows(), rows(), low(), low(), None if gate is None else rows())
    du, ddt, dB, dC, dgate = out
    assert (dgate is None) == (gate is None)
    z, ld_z = _opt_rows(dgate, u)
    f32 = lambda t, *s: torch.empty(s, dtype=torch.float32, device=dev) if t else None  # noqa: E731
    dA, dskip, dbias, dinitial = f32(True, ch, d.states), f32(skip is not None, ch), f32(dt_bias is not None, ch), f32(want_dinitial, *shape)
    address = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    rc = lib().spc_selective_scan_backward(d, dout.data_ptr(), _norm_rows(dout, u), *args, at, _f32(initial_state, shape, dev), _f32(dstate, shape, dev),
                                           du.data_ptr(), _norm_rows(du, u), ddt.data_ptr(), _norm_rows(ddt, u), dA.data_ptr(),
                                           _heads(dB, n, d.groups, d.states, u.dtype, dev), _heads(dC, n, d.groups, d.states, u.dtype, dev), address(dskip), z, ld_z,
                                           address(dbias), address(dinitial), current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return ScanGradients(du, ddt, dA, dB, dC, dskip, dgate, dbias, dinitial)


def spc_selective_scan_step(u: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, state: torch.Tensor,
                            skip: torch.Tensor | None = None, gate: torch.Tensor | None = None, dt_bias: torch.Tensor | None = None,
                            softplus: bool = True, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """One more row for every stream: u [streams, channels] and so on; state [streams, channels, states] fp32 is updated in place."""
    d, args, _ = _scan(u, dt, A, B, C, skip, gate, dt_bias, None, softplus)
    y = torch.empty(d.n_rows, d.channels, dtype=u.dtype, device=u.device) if out is None else out
    assert state is not None
    rc = lib().spc_selective_scan_step(d, *args, _f32(state, (d.n_rows, d.channels, d.states), u.device), y.data_ptr(),
                                       d.channels if out is None else _norm_rows(out, u), current_raw_stream() if stream is None else _stream(stream))
    if rc:
        _check(rc)
    return y


def spc_batch_offsets(keys: torch.Tensor, desc: PackDesc, n_batch: int, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """First row of every scene in sorted keys, and their end: int32 [n_batch + 1]."""
    assert keys.dim() == 1 and keys.dtype == (torch.int32 if desc.key_bits == 32 else torch.int64)
    if out is None:
        out = torch.empty(n_batch + 1, dtype=torch.int32, device=keys.device)
    assert out.dtype == torch.int32 and out.shape == (n_batch + 1,)
    _check(lib().spc_batch_offsets(_dev_ptr(keys), keys.shape[0], ctypes.byref(desc), n_batch, _dev_ptr(out), _stream(stream)))
    return out


def spc_probe_copy(src: torch.Tensor, dst: torch.Tensor, stream=None) -> int:
    """dst = src by the library's plain copy kernel; returns the bytes moved one way."""
    assert src.is_cuda and dst.is_cuda and src.is_contiguous() and dst.is_contiguous()
    nbytes = src.numel() * src.element_size()
    assert nbytes == dst.numel() * dst.element_size()
    _check(lib().spc_probe_copy(src.data_ptr(), dst.data_ptr(), nbytes, _stream(stream)))
    return nbytes


def spc_probe_mfma(iters: int, sink: torch.Tensor, stream=None) -> float:
    """Enqueues the register-resident MFMA loop; returns the floating-point operations of the launch."""
    flops = ctypes.c_double(0.0)
    _check(lib().spc_probe_mfma(int(iters), sink.data_ptr(), ctypes.byref(flops), _stream(stream)))
    return float(flops.value)


def spc_release_cache() -> None:
    _check(lib().spc_release_cache())
