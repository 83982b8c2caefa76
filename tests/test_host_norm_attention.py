"""What the calls of norms and attention refuse, through the C ABI without a GPU: every refusal comes before anything is enqueued."""
import ctypes

import pytest

from paper_2511_20834_amd import binding as B

P = 1 << 20  # (an address that nobody reads)
F32, F16 = B.DTYPE_F32, B.DTYPE_F16


def forward(x=P, ld_x=8, r=None, ld_r=8, eps=1e-5, y=P, ld_y=8, s=None, ld_s=8, mean=None, rstd=None, n=4, c=8, dtype=F32):
    return B.lib().spc_layer_norm_forward(x, ld_x, r, ld_r, None, None, eps, y, ld_y, s, ld_s, mean, rstd, n, c, dtype, None)


def backward(dy=P, x=P, ld_x=8, mean=P, rstd=P, e=None, ld_e=8, dx=P, n=4, c=8, dtype=F32):
    return B.lib().spc_layer_norm_backward(dy, 8, x, ld_x, mean, rstd, None, e, ld_e, dx, 8, None, None, n, c, dtype, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(y=None), dict(ld_x=7), dict(ld_y=0), dict(r=P), dict(s=P), dict(r=P, s=P, ld_r=7), dict(mean=P), dict(rstd=P), dict(eps=0.0),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(n=-1), dict(c=0), dict(dtype=3), dict(x=P + 2), dict(y=P + 1, dtype=F16)], ids=str)
def test_norm_refuses(bad):
    assert forward(**bad) == B.ERR_ARG


def test_norm_refuses_wide_rows_and_takes_none():
    assert forward(c=8193, ld_x=8193, ld_y=8193) == B.ERR_UNSUPPORTED and backward(c=8193) == B.ERR_UNSUPPORTED
    assert forward(x=None, y=None, n=0) == B.OK


@pytest.mark.parametrize("bad", [dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(ld_x=7), dict(e=P, ld_e=1), dict(dtype=-1), dict(n=-5)], ids=str)
def test_norm_gradient_refuses(bad):
    assert backward(**bad) == B.ERR_ARG


def desc(dtype=F16, scenes=1, rows=40, heads=4, kv=2, dk=16, dv=16, scale=0.25):
    return B.AttnDesc(dtype, scenes, rows, heads, kv, dk, dv, scale)


ROWS = B.AttnRows(P, 64, 16)


def attention(d=None, q=ROWS, k=ROWS, v=ROWS, g=P, at=None, out=ROWS):
    return B.lib().spc_linear_attention_forward(desc() if d is None else d, q, k, v, g, at, None, out, None, None)


@pytest.mark.parametrize("d", [desc(dtype=3), desc(scenes=0), desc(scenes=2), desc(rows=-1), desc(heads=0), desc(kv=0), desc(heads=3), desc(dk=0), desc(dv=0), desc(scale=float("nan")),
                               desc(scale=float("inf"))])
def test_attention_refuses_descriptors(d):
    assert attention(d) == B.ERR_ARG


@pytest.mark.parametrize("d", [desc(dk=129), desc(dv=200), desc(rows=1 << 31), desc(scenes=100_000)])
def test_attention_has_limits(d):
    assert attention(d, at=P) == B.ERR_UNSUPPORTED


@pytest.mark.parametrize("bad", [dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(g=None), dict(q=B.AttnRows(None, 64, 16)), dict(v=B.AttnRows(P + 1, 64, 16)), dict(k=B.AttnRows(P, -64, 16)),
                                 dict(q=B.AttnRows(P, 64, -1)), dict(out=B.AttnRows(P, 64, 15)), dict(out=B.AttnRows(P, 15, 64)), dict(out=B.AttnRows(P, 63, 16)), dict(out=B.AttnRows(P, 0, 16)),
                                 dict(out=B.AttnRows(P, 16, 600))], ids=lambda b: next(iter(b)))
def test_attention_refuses_rows(bad):
    assert attention(**bad) == B.ERR_ARG


def test_gradients_steps_and_offsets_refuse():
    L, d = B.lib(), desc()
    assert L.spc_linear_attention_backward(d, ROWS, ROWS, ROWS, ROWS, P, None, None, None, ROWS, ROWS, None, None, None) == B.ERR_ARG
    assert L.spc_linear_attention_backward(d, ROWS, ROWS, ROWS, ROWS, None, None, None, None, ROWS, ROWS, ROWS, None, None) == B.ERR_ARG
    assert L.spc_linear_attention_backward(d, ROWS, ROWS, ROWS, ROWS, P, None, None, None, B.AttnRows(P, 8, 16), ROWS, ROWS, None, None) == B.ERR_ARG
    assert L.spc_linear_attention_step(d, ROWS, ROWS, ROWS, P, None, ROWS, None) == B.ERR_ARG
    assert L.spc_linear_attention_step(desc(rows=0), None, None, None, P, None, None, None) == B.OK
    assert L.spc_linear_attention_step(desc(rows=1 << 23), ROWS, ROWS, ROWS, P, P, ROWS, None) == B.ERR_UNSUPPORTED
    p = B.spc_pack_desc_fit([0, 0, 0], [9, 9, 9], 2, 1, 1)
    for n, batch, keys, out in ((-1, 2, P, P), (5, 0, P, P), (5, 2, None, P), (5, 2, P, None), (5, (1 << 30) + 1, P, P), (1 << 31, 2, P, P)):
        assert L.spc_batch_offsets(keys, n, ctypes.byref(p), batch, out, None) == B.ERR_ARG
    assert L.spc_batch_offsets(P, 5, None, 2, P, None) == B.ERR_ARG
    assert "scenes" in B.lib().spc_last_error().decode() or "NULL" in B.lib().spc_last_error().decode()


@pytest.mark.parametrize("scenes", [0, -7, 100_000, 2 ** 31 - 1])
def test_steps_do_not_read_the_number_of_scenes(scenes):
    L = B.lib()
    assert L.spc_linear_attention_step(desc(rows=0, scenes=scenes), None, None, None, P, None, None, None) == B.OK
    assert L.spc_linear_attention_step(desc(scenes=scenes), ROWS, ROWS, ROWS, P, None, ROWS, None) == B.ERR_ARG  # (no state)
    assert L.spc_linear_attention_step(desc(scenes=scenes, heads=3), ROWS, ROWS, ROWS, P, P, ROWS, None) == B.ERR_ARG
    assert L.spc_linear_attention_step(desc(rows=1 << 23, scenes=scenes), ROWS, ROWS, ROWS, P, P, ROWS, None) == B.ERR_UNSUPPORTED
    assert L.spc_linear_attention_step(desc(rows=0, heads=300_000, kv=300_000), None, None, None, P, None, None, None) == B.OK
