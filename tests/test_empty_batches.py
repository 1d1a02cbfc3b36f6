"""Calls with no rows or no columns do nothing and succeed, whatever the leading dimensions: an empty tensor's address is null, so two
of them look like one, but that is no call in place."""

import ctypes as C

import pytest
import torch


def _L():
    from paper_2309_01226_amd import _lib
    return _lib


@pytest.mark.parametrize("rows,cols", [(0, 64), (9, 0), (0, 0)])
def test_dropout_of_nothing(rows, cols):
    L = _L()
    assert L.lib().sat_op_dropout(None, 64, None, 72, 0, rows, cols, 0.5, 1, None, None) == L.SAT_OK, L.last_error()


def test_boundary_of_nothing():
    L = _L()
    d = L.sat_residual_norm_desc(ldx=64, ldf=64, ldy=72, ldh=64, T=0, d=64, stream_f32=1, pre=1, post=2, alpha=1.0, beta=1.0, eps=1e-5)
    assert L.lib().sat_op_residual_norm_fwd(C.byref(d), None) == L.SAT_OK, L.last_error()


def test_boundary_backward_of_nothing():
    L = _L()
    d = L.sat_residual_norm_desc(ldf=64, ldy=64, lddy=72, lddh=64, lddx=64, lddf=64, T=0, d=64, stream_f32=1, pre=1, post=2, alpha=1.0, beta=1.0,
                                 eps=1e-5)
    assert L.lib().sat_op_residual_norm_bwd(C.byref(d), None) == L.SAT_OK, L.last_error()


def test_rotary_of_nothing():
    L = _L()
    assert L.lib().sat_op_rotary_axes(None, 64, None, 72, 0, None, 1, 1, (C.c_int32 * 1)(8), 0, 4, 16, 10000.0, 1, 0, 0, None) == L.SAT_OK, \
        L.last_error()


@pytest.mark.gpu
def test_empty_views():
    """As a program makes them: rows of a wider buffer, none of which is there."""
    from paper_2309_01226_amd import ops
    bf, f4 = torch.bfloat16, torch.float32
    wide = lambda dt: torch.empty(0, 80, dtype=dt, device="cuda")[:, :64]  # noqa: E731
    flat = lambda dt: torch.empty(0, 64, dtype=dt, device="cuda")  # noqa: E731
    ops.dropout(wide(bf), 0.5, 1, out=flat(bf))
    st, s = torch.empty(4, 0, device="cuda"), torch.full((64,), 7.0, device="cuda")
    ops.residual_norm_fwd(wide(f4), flat(bf), flat(f4), flat(bf), st, 64, pre="rms", post="layer")
    ops.residual_norm_bwd(wide(f4), flat(bf), flat(f4), flat(bf), st, flat(f4), flat(bf), 64, pre="rms", post="layer", dg_pre=s)
    ops.rotary_axes(wide(bf), torch.empty(0, 1, dtype=torch.int32, device="cuda"), 4, 16, [8], out=flat(bf))
    assert not s.any()
