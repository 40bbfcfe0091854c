"""Outputs in an input's place: what the C entry points of the operators around the GEMMs refuse, before anything is enqueued.

The pointers are never followed: every call here is refused, or has nothing to do.
"""
import ctypes

import pytest

from test_operator_refusals import BACKWARD, BF16, E4M3, EINVAL, F32, LinearArgs, NORM, OK, P, call, lib, linear, made, rms_norm
from test_operator_refusals import rms_norm_backward

APART = dict(x=P, r=2 * P, w=3 * P, y=4 * P, h=5 * P, inv=6 * P)


@pytest.mark.parametrize("change", [
    dict(y_dtype=E4M3, scales=7 * P, y=P), dict(y_dtype=E4M3, scales=7 * P, y=2 * P),       # 8-bit rows over other rows
    dict(y_dtype=E4M3, scales=7 * P, y=P, rows=1), dict(y_dtype=E4M3, scales=7 * P, y=5 * P),
    dict(y=P, ldy=104), dict(y=2 * P, ldr=104), dict(h=P, ldx=101), dict(h=2 * P, ldh=200), dict(y=5 * P)])
def test_norm(change):
    assert call(rms_norm, NORM, **{**APART, **change, "rows": 0}) == OK       # nothing is read or written
    assert call(rms_norm, NORM, **{**APART, "rows": 5, **change}) == EINVAL


@pytest.mark.parametrize("change", [dict(dx=2 * P, lddx=104), dict(dx=3 * P, ldh=104), dict(dx=4 * P, ldds=101)])
def test_norm_backward(change):
    apart = dict(dy=2 * P, h=3 * P, ds=4 * P, w=5 * P, inv=6 * P, dx=7 * P, dw=8 * P, ws=9 * P)
    assert call(rms_norm_backward, BACKWARD, **{**apart, **change}) == EINVAL


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("change", [dict(residual=4 * P, ldr=208), dict(preact=4 * P), dict(preact=4 * P, act=1),
                                    dict(preact=4 * P, act=2, act_grad=1, ldz=208)])
def test_linear(dtype, change):
    plan = made(300, 200, 512, dtype)
    a = LinearArgs(A=P, B=2 * P, C=4 * P, lda=512, ldb=512, ldr=200, ldz=200, ldc=200, transB=1, dtype=dtype, out_dtype=BF16)
    if dtype == E4M3:
        a.scale_a, a.scale_b = 5 * P, 6 * P
    for name, value in change.items():
        setattr(a, name, value)
    assert linear(plan, ctypes.byref(a), None) == EINVAL
    lib.cleave_plan_destroy(plan)
