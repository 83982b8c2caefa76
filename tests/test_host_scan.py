"""What the calls of root-mean-square norms, 8-bit products, causal convolution and selective scan refuse, through the C ABI without a GPU: every refusal comes before anything is
enqueued."""
import pytest

from paper_2511_20834_amd import binding as B

P = 1 << 20  # (an address that nobody reads)
F32, F16 = B.DTYPE_F32, B.DTYPE_F16
BIG = 1 << 31


def rms(x=P, ld_x=8, r=None, ld_r=8, eps=1e-5, y=P, ld_y=8, s=None, ld_s=8, n=4, c=8, dtype=F32):
    return B.lib().spc_rms_norm_forward(x, ld_x, r, ld_r, None, eps, y, ld_y, s, ld_s, None, n, c, dtype, None)


def rms8(x=P, ld_x=8, r=None, ld_r=8, eps=1e-5, y=P, ld_y=8, scale=P, s=None, ld_s=8, n=4, c=8, dtype=F32):
    return B.lib().spc_rms_norm_quantize(x, ld_x, r, ld_r, None, eps, y, ld_y, scale, s, ld_s, None, n, c, dtype, None)


NORM = [dict(x=None), dict(y=None), dict(ld_x=7), dict(ld_y=0), dict(r=P), dict(s=P), dict(r=P, s=P, ld_r=7), dict(r=P, s=P, ld_s=7), dict(eps=0.0), dict(eps=float("nan")),
        dict(eps=float("inf")), dict(n=-1), dict(c=0), dict(dtype=3), dict(x=P + 2)]


@pytest.mark.parametrize("bad", NORM + [dict(y=P + 1, dtype=F16)], ids=str)
def test_norm_refuses(bad):
    assert rms(**bad) == B.ERR_ARG


@pytest.mark.parametrize("bad", NORM + [dict(scale=None)], ids=str)
def test_norm_to_8_bits_refuses(bad):
    assert rms8(**bad) == B.ERR_ARG


def test_norms_refuse_wide_rows_and_take_none():
    L = B.lib()
    assert rms(c=8193, ld_x=8193, ld_y=8193) == rms8(c=8193, ld_x=8193, ld_y=8193) == B.ERR_UNSUPPORTED
    assert rms(x=None, y=None, n=0) == rms8(x=None, y=None, scale=None, n=0) == B.OK
    assert L.spc_quantize_rows(P, 8193, P, 8193, P, 4, 8193, F32, None) == B.ERR_UNSUPPORTED
    assert L.spc_quantize_rows(None, 8, None, 8, None, 0, 8, F32, None) == B.OK


@pytest.mark.parametrize("bad", [(None, 8, P, 8, P, 4, 8, F32), (P, 8, None, 8, P, 4, 8, F32), (P, 8, P, 8, None, 4, 8, F32), (P, 7, P, 8, P, 4, 8, F32), (P, 8, P, 7, P, 4, 8, F32),
                                 (P, 8, P, 8, P, -1, 8, F32), (P, 8, P, 8, P, 4, 0, F32), (P, 8, P, 8, P, 4, 8, 9), (P + 1, 8, P, 8, P, 4, 8, F16)], ids=str)
def test_rows_in_8_bits_refuse(bad):
    assert B.lib().spc_quantize_rows(*bad, None) == B.ERR_ARG


def rms_back(dy=P, ld_dy=8, x=P, ld_x=8, rstd=P, e=None, ld_e=8, dx=P, ld_dx=8, n=4, c=8, dtype=F32):
    return B.lib().spc_rms_norm_backward(dy, ld_dy, x, ld_x, rstd, None, e, ld_e, dx, ld_dx, None, n, c, dtype, None)


@pytest.mark.parametrize("bad", [dict(dy=None), dict(x=None), dict(dx=None), dict(rstd=None), dict(ld_dy=7), dict(ld_x=7), dict(ld_dx=1), dict(e=P, ld_e=1), dict(dtype=-1), dict(n=-5), dict(c=0)],
                         ids=str)
def test_norm_gradient_refuses(bad):
    assert rms_back(**bad) == B.ERR_ARG
    assert rms_back(c=8193) == B.ERR_UNSUPPORTED


def linear(x=P, ld_x=16, sx=P, w=P, ld_w=16, sw=P, out=P, ld_out=32, n=4, c=16, m=32, dtype=F16):
    return B.lib().spc_linear_f8(x, ld_x, sx, w, ld_w, sw, out, ld_out, n, c, m, dtype, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(sx=None), dict(w=None), dict(sw=None), dict(out=None), dict(ld_x=15), dict(ld_w=15), dict(ld_out=31), dict(n=-1), dict(c=0), dict(m=0), dict(dtype=3),
                                 dict(out=P + 1), dict(out=P + 2, dtype=F32)], ids=str)
def test_product_refuses(bad):
    assert linear(**bad) == B.ERR_ARG


def test_product_has_limits():
    assert linear(c=65537, ld_x=65537, ld_w=65537) == linear(m=65537, ld_out=65537) == linear(n=(1 << 30) + 1) == B.ERR_UNSUPPORTED
    assert linear(x=None, n=0) == B.OK


def conv(x=P, ld_x=8, w=P, width=4, at=None, scenes=1, rows_in=None, y=P, ld_y=8, rows_out=None, n=4, c=8, dtype=F16):
    return B.lib().spc_causal_conv_forward(x, ld_x, w, None, width, 1, at, scenes, rows_in, y, ld_y, rows_out, n, c, dtype, None)


def conv_back(x=P, ld_x=8, w=P, width=4, at=None, scenes=1, rows_in=None, y=P, ld_y=8, rows_out=None, dy=P, drows=None, n=4, c=8, dtype=F16):
    return B.lib().spc_causal_conv_backward(dy, 8, x, ld_x, w, None, width, 1, at, scenes, rows_in, drows, y, ld_y, None, None, rows_out, n, c, dtype, None)


@pytest.mark.parametrize("call", [conv, conv_back])
@pytest.mark.parametrize("bad", [dict(x=None), dict(w=None), dict(y=None), dict(ld_x=7), dict(ld_y=7), dict(width=0), dict(scenes=0), dict(scenes=2), dict(n=-1), dict(c=0), dict(dtype=7), dict(x=P + 1), dict(y=P + 1),
                                 dict(rows_in=P + 1), dict(rows_out=P + 1)], ids=str)
def test_convolution_refuses(bad, call):
    assert call(**bad) == B.ERR_ARG


def test_convolution_refuses_shared_states_and_has_limits():
    assert conv(rows_in=P, rows_out=P) == conv_back(drows=P, rows_out=P) == conv_back(dy=None) == conv_back(drows=P + 1) == B.ERR_ARG
    for call in (conv, conv_back):
        assert call(width=5) == call(c=65537, ld_x=65537, ld_y=65537) == call(n=BIG) == call(n=BIG - 65535) == call(at=P, scenes=200_001) == B.ERR_UNSUPPORTED
    assert conv(c=65536, ld_x=65536, ld_y=65536, at=P, scenes=200_000, n=10) == B.ERR_UNSUPPORTED  # (a launch takes less than 2^32 threads)
    assert conv(x=None, y=None, n=0) == B.OK


def conv_step(x=P, ld_x=8, w=P, width=4, rows=P, y=P, ld_y=8, n=4, c=8, dtype=F16):
    return B.lib().spc_causal_conv_step(x, ld_x, w, None, width, 1, rows, y, ld_y, n, c, dtype, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(w=None), dict(rows=None), dict(y=None), dict(ld_x=7), dict(ld_y=7), dict(width=0), dict(n=-1), dict(c=0), dict(dtype=7), dict(rows=P + 1)], ids=str)
def test_convolution_step_refuses(bad):
    assert conv_step(**bad) == B.ERR_ARG
    assert conv_step(width=5) == conv_step(n=BIG + 1) == B.ERR_UNSUPPORTED
    assert conv_step(x=None, rows=None, n=0) == B.OK


def desc(dtype=F16, scenes=1, rows=40, channels=64, groups=2, states=16, softplus=1):
    return B.ScanDesc(dtype, scenes, rows, channels, groups, states, softplus)


LOW = B.AttnRows(P, 32, 16)


def scan(d=None, u=P, ld_u=64, dt=P, ld_dt=64, A=P, b=LOW, c=LOW, z=None, ld_z=64, at=None, s_in=None, out=P, ld_out=64, s_out=None):
    return B.lib().spc_selective_scan_forward(desc() if d is None else d, u, ld_u, dt, ld_dt, A, b, c, None, z, ld_z, None, at, s_in, out, ld_out, s_out, None)


def scan_back(d=None, u=P, ld_u=64, dt=P, ld_dt=64, A=P, b=LOW, c=LOW, z=None, ld_z=64, at=None, s_in=None, out=P, ld_out=64, s_out=None, dout=P, ddt=P, db=LOW, dc=LOW, dz=None, ds=None):
    return B.lib().spc_selective_scan_backward(desc() if d is None else d, dout, ld_out, u, ld_u, dt, ld_dt, A, b, c, None, z, ld_z, None, at, s_in, ds, out, ld_out, ddt, ld_out, None, db, dc, None, dz, 64,
                                               None, s_out, None)


def scan_step(d=None, u=P, ld_u=64, dt=P, ld_dt=64, A=P, b=LOW, c=LOW, z=None, ld_z=64, out=P, ld_out=64, state=P):
    return B.lib().spc_selective_scan_step(desc() if d is None else d, u, ld_u, dt, ld_dt, A, b, c, None, z, ld_z, None, state, out, ld_out, None)


@pytest.mark.parametrize("call", [scan, scan_back, scan_step])
@pytest.mark.parametrize("bad", [dict(u=None), dict(dt=None), dict(A=None), dict(b=None), dict(c=None), dict(out=None), dict(ld_u=63), dict(ld_dt=63), dict(ld_out=63), dict(z=P, ld_z=63), dict(u=P + 1),
                                 dict(z=P + 1), dict(b=B.AttnRows(None, 32, 16)), dict(c=B.AttnRows(P + 1, 32, 16)), dict(b=B.AttnRows(P, -1, 16)), dict(c=B.AttnRows(P, 32, -16)),
                                 dict(b=B.AttnRows(P, 1 << 40, 16))], ids=lambda b: "-".join(b))
def test_scan_refuses(bad, call):
    assert call(**bad) == B.ERR_ARG


@pytest.mark.parametrize("call", [scan, scan_back, scan_step])
@pytest.mark.parametrize("d", [desc(dtype=3), desc(rows=-1), desc(channels=0), desc(groups=0), desc(groups=3), desc(states=0)])
def test_scan_refuses_descriptors(d, call):
    assert call(d) == B.ERR_ARG


def test_scan_has_limits():
    wide = dict(ld_u=1 << 17, ld_dt=1 << 17, ld_out=1 << 17)
    for call in (scan, scan_back, scan_step):
        assert call(desc(states=65)) == call(desc(channels=65_538), **wide) == B.ERR_UNSUPPORTED
    for call in (scan, scan_back):
        assert call(desc(scenes=0)) == call(desc(scenes=2)) == B.ERR_ARG
        assert call(desc(rows=BIG), at=P) == call(desc(scenes=200_001), at=P) == call(desc(scenes=200_000, channels=65_536), at=P, **wide) == B.ERR_UNSUPPORTED
    assert scan_step(desc(rows=1 << 24), ) == B.ERR_UNSUPPORTED
    # (five states count as eight)
    assert scan_step(desc(rows=1 << 28, channels=1, groups=1, states=5)) == scan_step(desc(rows=(1 << 28) // 3 + 1, channels=3, groups=1, states=5)) == B.ERR_UNSUPPORTED
    assert scan_step(desc(rows=0, scenes=-3), u=None, state=None) == scan(desc(rows=0), u=None, out=None) == B.OK


def test_scan_refuses_states_and_gradients():
    assert scan(s_in=P, s_out=P) == scan_back(ds=P, s_out=P) == scan_step(state=None) == B.ERR_ARG
    assert scan_back(dout=None) == scan_back(ddt=None) == scan_back(db=None) == scan_back(dc=None) == scan_back(z=P) == B.ERR_ARG
    # (every row and group of an output has places of its own)
    for low in (B.AttnRows(P, 0, 16), B.AttnRows(P, 32, 0), B.AttnRows(P, 31, 16), B.AttnRows(P, 16, 600)):
        assert scan_back(db=low) == scan_back(dc=low) == B.ERR_ARG


def test_scan_counts_states_of_all_scenes():
    """2^29 of them, counted as powers of two, are too many (a chain of segments takes a lane for each)."""
    for call in (scan, scan_back):
        assert call(desc(scenes=1 << 16, channels=512, groups=1, states=16), at=P, ld_u=512, ld_dt=512, ld_out=512) == B.ERR_UNSUPPORTED
        assert call(desc(scenes=1 << 16, channels=512, groups=1, states=9), at=P, ld_u=512, ld_dt=512, ld_out=512) == B.ERR_UNSUPPORTED


def test_limits_of_launches():
    """Groups of one channel take a wave each; what a launch does not hold is refused before anything is enqueued."""
    one = B.AttnRows(P, 512, 1)
    many = dict(at=P, ld_u=512, ld_dt=512, ld_out=512, b=one, c=one)
    assert scan_back(desc(scenes=60_000, channels=512, groups=512, states=1), **many, db=one, dc=one) == B.ERR_UNSUPPORTED  # (scenes x channels to 64 each: 2^30.9)
    assert scan(desc(scenes=200_000, channels=512, groups=512, states=1), **many) == B.ERR_UNSUPPORTED
    assert conv(c=65536, ld_x=65536, ld_y=65536, at=P, scenes=200_000, n=10, dtype=F32) == B.ERR_UNSUPPORTED
    assert conv_step(n=(1 << 30) + 1, c=9, ld_x=9, ld_y=9) == conv_step(n=(1 << 29) + 1, c=13, ld_x=13, ld_y=13, dtype=F32) == B.ERR_UNSUPPORTED
