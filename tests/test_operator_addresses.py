"""Vectors and workspaces in another one's place: what the C entry points of the norm, the bias gradient and the linear product refuse,
before anything is enqueued (the pointers are never followed)."""
import ctypes

import pytest

from test_operator_refusals import BACKWARD, BF16, BIAS, E4M3, EINVAL, F32, LinearArgs, NORM, OK, P, bias_grad, call, lib, linear, made
from test_operator_refusals import rms_norm, rms_norm_backward

APART = {**NORM, **dict(x=P, r=2 * P, w=3 * P, y=4 * P, h=5 * P, inv=6 * P, y_dtype=E4M3, scales=7 * P)}
BACK = {**BACKWARD, **dict(dy=P, h=2 * P, ds=3 * P, w=4 * P, inv=5 * P, dx=6 * P, dw=7 * P, ws=8 * P)}


@pytest.mark.parametrize("change", [
    dict(inv=7 * P), dict(inv=3 * P), dict(inv=4 * P), dict(inv=5 * P), dict(inv=P), dict(inv=2 * P), dict(scales=3 * P), dict(scales=4 * P),
    dict(scales=5 * P), dict(scales=P), dict(y=3 * P), dict(h=3 * P)])
def test_norm(change):
    assert call(rms_norm, APART, **change) == OK       # no rows
    assert call(rms_norm, APART, **{"rows": 5, **change}) == EINVAL


@pytest.mark.parametrize("change", [
    dict(dw=8 * P), dict(dw=6 * P), dict(dx=8 * P), dict(dx=4 * P), dict(dx=5 * P), dict(ws=P), dict(ws=2 * P), dict(ws=3 * P),
    dict(ws=4 * P), dict(ws=5 * P)])
def test_norm_backward(change):
    assert call(rms_norm_backward, BACK, **change) == EINVAL


@pytest.mark.parametrize("change", [dict(db=3 * P), dict(ws=P), dict(db=P)])
def test_bias_grad(change):
    assert call(bias_grad, {**BIAS, **dict(rows=100000, dy=P, db=2 * P, ws=3 * P)}, **change) == EINVAL


@pytest.mark.parametrize("M,N,K,dtype", [(64, 512, 11008, BF16), (1, 512, 4096, BF16), (64, 512, 4096, F32)])
@pytest.mark.parametrize("change", [dict(partials=n * P) for n in range(1, 7)] +
                         [dict(C=P), dict(C=2 * P), dict(preact=P), dict(preact=2 * P), dict(C=3 * P), dict(preact=3 * P)])
def test_linear(M, N, K, dtype, change):
    """The workspace of a split product, and outputs in an operand's or the bias's place."""
    plan = made(M, N, K, dtype)
    a = LinearArgs(A=P, B=2 * P, bias=3 * P, residual=4 * P, preact=5 * P, C=6 * P, partials=7 * P, lda=K, ldb=K, ldr=N, ldz=N, ldc=N,
                   transB=1, dtype=dtype, out_dtype=dtype)
    for name, value in change.items():
        setattr(a, name, value)
    assert lib.cleave_linear_workspace(plan) > 0
    assert linear(plan, ctypes.byref(a), None) == EINVAL
    lib.cleave_plan_destroy(plan)
