"""What the C entry points of the operators around the GEMMs refuse, before anything is enqueued.

The pointers are never followed: every call here is refused, or has nothing to do.
"""
import ctypes
import math

import pytest

import paper_2512_22142_amd as cleave
from paper_2512_22142_amd.binding import LIB_PATH

F32, BF16, E4M3 = 0, 1, 2
OK, EINVAL = 0, -1
P = 1 << 20          # an address on every boundary
i64, i32, p, c_int, f32, f64 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_double

lib = ctypes.CDLL(LIB_PATH)


def declare(name, args, res=c_int):
    f = getattr(lib, name)
    f.argtypes, f.restype = args, res
    return f


rms_norm = declare("cleave_rms_norm", [i64, i64, p, i64, p, i64, c_int, p, f32, p, i64, c_int, p, p, i64, p, p])
rms_norm_backward = declare("cleave_rms_norm_backward", [i64, i64, p, i64, p, i64, p, i64, c_int, p, p, p, i64, p, p, p])
bias_grad = declare("cleave_bias_grad", [i64, i64, p, i64, c_int, p, p, p])
adamw = declare("cleave_adamw", [i64, p, p, p, c_int, p, p, p, p, p, p, f64, f64, f64, f64, f64, i64, p])
norm_ws = declare("cleave_rms_norm_workspace", [i64, i64], i64)
bias_ws = declare("cleave_bias_grad_workspace", [i64, i64], i64)
plan_linear = declare("cleave_plan_linear", [i64, i64, i64, c_int, p])
linear_ws = declare("cleave_linear_workspace", [p], i64)


class LinearArgs(ctypes.Structure):
    _fields_ = ([(n, p) for n in ("A", "B", "scale_a", "scale_b", "bias", "residual", "preact", "C", "partials")] +
                [(n, i64) for n in ("lda", "ldb", "ldr", "ldz", "ldc")] +
                [(n, i32) for n in ("transA", "transB", "dtype", "out_dtype", "act", "act_grad")])


linear = declare("cleave_linear", [p, ctypes.POINTER(LinearArgs), p])


def call(f, base, **change):
    return f(*{**base, **change}.values())


NORM = dict(rows=0, cols=100, x=P, ldx=100, r=P, ldr=100, dtype=BF16, w=P, eps=1e-5, y=P, ldy=100, y_dtype=BF16, scales=None,
            h=P, ldh=100, inv=P, stream=None)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(cols=0), dict(rows=2 ** 31), dict(cols=2 ** 31, ldx=2 ** 32, ldr=2 ** 32, ldy=2 ** 32, ldh=2 ** 32),
    dict(dtype=E4M3, y_dtype=E4M3, scales=P), dict(dtype=7, y_dtype=7), dict(y_dtype=F32), dict(y_dtype=E4M3), dict(scales=P),
    dict(x=None), dict(w=None), dict(y=None), dict(ldx=99), dict(ldr=99), dict(ldy=99), dict(ldh=99), dict(x=P + 1), dict(r=P + 1),
    dict(y=P + 1), dict(h=P + 1), dict(w=P + 2), dict(inv=P + 2), dict(eps=-1e-6), dict(eps=math.inf), dict(eps=math.nan),
    dict(dtype=F32, y_dtype=F32, x=P + 2)])
def test_norm(change):
    assert call(rms_norm, NORM) == OK
    assert call(rms_norm, NORM, r=None, ldr=0, h=None, ldh=0, inv=None) == OK
    assert call(rms_norm, NORM, y_dtype=E4M3, scales=P, y=P + 1) == OK
    assert call(rms_norm, NORM, **change) == EINVAL


BACKWARD = dict(rows=5, cols=100, dy=P, lddy=100, h=P, ldh=100, ds=P, ldds=100, dtype=BF16, w=P, inv=P, dx=P, lddx=100, dw=P, ws=P,
                stream=None)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(cols=0), dict(dtype=E4M3), dict(dy=None), dict(h=None), dict(w=None), dict(inv=None), dict(dx=None), dict(dw=None),
    dict(ws=None), dict(lddy=99), dict(ldh=99), dict(ldds=99), dict(lddx=99), dict(dy=P + 1), dict(ds=P + 1), dict(ws=P + 2)])
def test_norm_backward(change):
    assert call(rms_norm_backward, BACKWARD, **change) == EINVAL


BIAS = dict(rows=5, cols=100, dy=P, ld=100, dtype=BF16, db=P, ws=P, stream=None)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(cols=0), dict(dtype=E4M3), dict(dy=None), dict(db=None), dict(ws=None),
                                    dict(ld=99), dict(dy=P + 1), dict(db=P + 2)])
def test_bias_grad(change):
    assert call(bias_grad, BIAS, **change) == EINVAL


def test_workspaces():
    for f in (norm_ws, bias_ws):
        assert f(-1, 8) == EINVAL and f(8, 0) == EINVAL and f(2 ** 31, 8) == EINVAL and f(8, 2 ** 31) == EINVAL
        for rows, cols in ((0, 8), (1, 1), (5000, 4096), (2 ** 31 - 1, 2 ** 31 - 1)):
            assert f(rows, cols) >= cols and f(rows, cols) % cols == 0


def pointers(*values):
    return ctypes.cast((p * len(values))(*values), p)


def adam(**change):
    sizes = change.pop("sizes", (0, 0))
    base = dict(n=2, sizes=ctypes.cast((i64 * len(sizes))(*sizes), p), w=pointers(P, P), g=pointers(P, P), g_dtype=BF16,
                m=pointers(P, P), v=pointers(P, P), ms=None, vs=None, copy=None, gs=None, lr=1e-3, b1=0.9, b2=0.95, eps=1e-8, wd=0.1,
                step=1, stream=None)
    return call(adamw, base, **change)


@pytest.mark.parametrize("change", [
    dict(n=-1), dict(sizes=(0, -1)), dict(sizes=(0, 2 ** 40)), dict(w=None), dict(g=None), dict(m=None), dict(v=None), dict(g_dtype=E4M3),
    dict(ms=pointers(P, P)), dict(vs=pointers(P, P)), dict(step=0), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=math.nan),
    dict(eps=-1e-9), dict(eps=math.nan), dict(lr=math.nan), dict(wd=math.nan), dict(gs=P + 2),
    dict(sizes=(0, 5), w=pointers(P, None)), dict(sizes=(5, 0), w=pointers(P + 2, None)), dict(sizes=(5, 0), g=pointers(P + 1, P)),
    dict(sizes=(5, 0), m=pointers(P + 2, P)), dict(sizes=(5, 0), copy=pointers(None, None)),
    dict(sizes=(5, 0), ms=pointers(None, P), vs=pointers(P, P)), dict(sizes=(5, 0), ms=pointers(P, P), vs=pointers(P + 1, P))])
def test_adamw(change):
    assert adam() == OK and adam(n=0, sizes=(), w=None, g=None, m=None, v=None) == OK
    assert adam(w=pointers(None, None), ms=pointers(None, None), vs=pointers(None, None)) == OK   # empty tensors
    assert adam(**change) == EINVAL


def made(M, N, K, dtype):
    plan = p()
    assert plan_linear(M, N, K, dtype, ctypes.byref(plan)) == OK
    return plan


def test_plans():
    plan = p()
    for args in ((0, 8, 8, BF16), (8, 0, 8, BF16), (8, 8, 0, BF16), (8, 8, 8, 3), (8, 8, 8, -1), (2 ** 31, 8, 8, BF16), (8, 8, 24, E4M3)):
        assert plan_linear(*args, ctypes.byref(plan)) == EINVAL and not plan.value
    assert plan_linear(8, 8, 8, BF16, None) == EINVAL
    assert linear_ws(None) == EINVAL
    batched = cleave.plan_batched(8, 8, 8, 8, 8, 1, 2)
    assert linear_ws(batched._h) == EINVAL
    for M, N, K, dtype in ((1, 512, 4096, BF16), (64, 512, 11008, BF16), (4096, 4096, 4096, BF16), (1, 64, 16384, E4M3), (64, 512, 4096, F32)):
        made_plan = made(M, N, K, dtype)
        floats = linear_ws(made_plan)
        assert floats % (M * N) == 0 and floats // (M * N) != 1      # none, or at least two splits' blocks
        lib.cleave_plan_destroy(made_plan)


@pytest.fixture(scope="module")
def plans():
    some = {d: made(300, 200, 512, d) for d in (F32, BF16, E4M3)}
    some["split"] = made(64, 512, 11008, BF16)
    yield some
    for plan in some.values():
        lib.cleave_plan_destroy(plan)


def args_of(dtype):
    a = LinearArgs(A=P, B=P, C=P, lda=512, ldb=512, ldr=200, ldz=200, ldc=200, transB=1, dtype=dtype, out_dtype=BF16)
    if dtype == E4M3:
        a.scale_a = a.scale_b = P
    return a


@pytest.mark.parametrize("dtype,change", [
    *[(d, c) for d in (F32, BF16, E4M3) for c in (
        dict(A=None), dict(B=None), dict(C=None), dict(lda=511), dict(ldb=511), dict(ldc=199), dict(residual=P, ldr=199),
        dict(preact=P, ldz=199), dict(C=P + 1), dict(residual=P + 1), dict(preact=P + 1), dict(bias=P + 2), dict(transA=2), dict(transB=-1),
        dict(out_dtype=E4M3), dict(act=4), dict(act=-1), dict(act_grad=2), dict(act_grad=1, act=1), dict(act_grad=1, bias=P),
        dict(dtype=3))],
    (BF16, dict(A=P + 1)), (F32, dict(B=P + 2)), (BF16, dict(scale_a=P)), (F32, dict(scale_b=P)), (BF16, dict(dtype=E4M3)),
    (BF16, dict(transB=0, ldb=199)), (BF16, dict(transA=1, lda=299)), (F32, dict(out_dtype=F32, C=P + 2)),
    (E4M3, dict(scale_a=None)), (E4M3, dict(scale_b=None)), (E4M3, dict(transB=0)), (E4M3, dict(transA=1)), (E4M3, dict(A=P + 8)),
    (E4M3, dict(B=P + 8)), (E4M3, dict(lda=520)), (E4M3, dict(ldb=520)), (E4M3, dict(lda=1 << 22)), (E4M3, dict(dtype=BF16)),
    (E4M3, dict(scale_a=P + 2))])
def test_linear(plans, dtype, change):
    a = args_of(dtype)
    for name, value in change.items():
        setattr(a, name, value)
    assert linear(plans[dtype], ctypes.byref(a), None) == EINVAL


def test_linear_without_its_workspace(plans):
    a = LinearArgs(A=P, B=P, C=P, lda=11008, ldb=11008, ldc=512, transB=1, dtype=BF16, out_dtype=BF16)
    assert linear_ws(plans["split"]) > 0
    assert linear(plans["split"], ctypes.byref(a), None) == EINVAL
    assert linear(None, ctypes.byref(a), None) == EINVAL and linear(plans[BF16], None, None) == EINVAL


def test_a_plan_of_8bit_operands_is_no_other_calls(plans):
    execute = declare("cleave_execute", [p, p, i64, p, i64, c_int, p, i64, c_int, c_int, p, p])
    reduce = declare("cleave_reduce", [p, p, p, i64, c_int, p])
    verify = declare("cleave_verify", [p, p, i64, c_int, p, i64, c_int, c_int, p, p, p, f64, p, p, p, p, p])
    for dtype in (F32, BF16):
        assert execute(plans[E4M3], None, 0, P, 512, 0, P, 512, 1, dtype, P, None) == EINVAL
        assert verify(plans[E4M3], P, 512, 0, P, 512, 1, dtype, P, P, P, 1e-3, None, None, None, P, None) == EINVAL
    assert reduce(plans[E4M3], P, P, 200, F32, None) == EINVAL
