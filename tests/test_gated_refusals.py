"""What the C entry points of the gated product refuse, before anything is enqueued (the pointers are never followed)."""
import ctypes

import pytest

from test_operator_refusals import BF16, E4M3, EINVAL, F32, OK, P, c_int, declare, i32, i64, lib, made, p

plan_gated = declare("cleave_plan_gated", [i64, i64, i64, c_int, p])
workspace = declare("cleave_gated_workspace", [p, c_int], i64)
grad_workspace = declare("cleave_gated_grad_workspace", [p, c_int], i64)


class Args(ctypes.Structure):
    _fields_ = ([(n, p) for n in ("A", "B_gate", "B_up", "scale_a", "scale_gate", "scale_up", "bias_gate", "bias_up", "gate", "up",
                                  "C", "partials")] +
                [(n, i64) for n in ("lda", "ldb", "ld_gate", "ld_up", "ldc")] +
                [(n, i32) for n in ("transB", "dtype", "out_dtype", "act")])


class GradArgs(ctypes.Structure):
    _fields_ = ([(n, p) for n in ("A", "B", "gate", "up", "dgate", "dup", "partials")] +
                [(n, i64) for n in ("lda", "ldb", "ld_gate", "ld_up", "ld_dgate", "ld_dup")] +
                [(n, i32) for n in ("transB", "dtype", "out_dtype", "act")])


gated = declare("cleave_linear_gated", [p, ctypes.POINTER(Args), p])
grad = declare("cleave_linear_gated_grad", [p, ctypes.POINTER(GradArgs), p])
declare("cleave_plan_partial_elems", [p], i64)


def gated_plan(M, N, K, dtype):
    out = p()
    assert plan_gated(M, N, K, dtype, ctypes.byref(out)) == OK
    return out


@pytest.mark.parametrize("args", [(0, 8, 8, BF16), (8, 0, 8, BF16), (8, 8, 0, BF16), (8, 8, 8, 3), (8, 8, 24, E4M3),
                                  (2 ** 31, 8, 8, BF16), (8, 2 ** 30, 8, BF16), (8, 8, 2 ** 31, BF16)])
def test_plan(args):
    out = p()
    assert plan_gated(*args, ctypes.byref(out)) == EINVAL and not out.value


def test_workspace():
    for dtype in (F32, BF16, E4M3):
        plan = gated_plan(300, 200, 512, dtype)
        some = lib.cleave_plan_partial_elems(plan)
        assert some % (2 * 300 * 200) == 0 and some > 0
        assert workspace(plan, 1) == (some if dtype == F32 else 0)
        assert workspace(plan, 0) == some if dtype == F32 else workspace(plan, 0) >= (0 if dtype == E4M3 else 1)
        assert dtype != E4M3 or workspace(plan, 0) == 0
        assert workspace(plan, 2) == EINVAL and workspace(None, 0) == EINVAL and grad_workspace(plan, 0) == EINVAL
        lib.cleave_plan_destroy(plan)
    one = gated_plan(1, 11008, 4096, BF16)
    assert workspace(one, 0) == 0 and workspace(one, 1) == 0
    lib.cleave_plan_destroy(one)
    narrow = gated_plan(2, 256, 8192, BF16)      # few columns: K is split
    assert workspace(narrow, 0) > 0 and workspace(narrow, 0) % (2 * 2 * 256) == 0 and workspace(narrow, 0) == workspace(narrow, 1)
    lib.cleave_plan_destroy(narrow)
    for dtype in (F32, BF16):
        plan = made(300, 200, 512, dtype)
        some = lib.cleave_plan_partial_elems(plan)
        assert some % (300 * 200) == 0 and some > 0 and workspace(plan, 0) == EINVAL
        assert grad_workspace(plan, 0) > 0 and grad_workspace(plan, 1) == (some if dtype == F32 else 0)
        lib.cleave_plan_destroy(plan)


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("change", [
    dict(A=None), dict(B_gate=None), dict(B_up=None), dict(C=None), dict(lda=511), dict(ldb=511), dict(ldc=199), dict(ld_gate=199),
    dict(ld_up=199), dict(transB=2), dict(dtype=7), dict(out_dtype=E4M3), dict(act=-1), dict(act=4), dict(C=4 * P + 1), dict(gate=P + 1),
    dict(bias_gate=P + 2), dict(bias_up=P + 1), dict(partials=P + 2), dict(gate=4 * P), dict(up=4 * P), dict(up=5 * P),
    dict(transB=0, ldb=199), dict(scale_gate="other"), dict(scale_a="other"), dict(C=P), dict(gate=2 * P), dict(up=3 * P)])
def test_gated(dtype, change):
    plan = gated_plan(300, 200, 512, dtype)
    a = Args(A=P, B_gate=2 * P, B_up=3 * P, C=4 * P, gate=5 * P, up=6 * P, bias_gate=7 * P, bias_up=8 * P, partials=9 * P, lda=512, ldb=512,
             ldc=200, ld_gate=200, ld_up=200, transB=1, dtype=dtype, out_dtype=BF16, act=3)
    if dtype == E4M3:
        a.scale_a, a.scale_gate, a.scale_up = 10 * P, 11 * P, 12 * P
    for name, value in change.items():
        setattr(a, name, (None if dtype == E4M3 else P) if value == "other" else value)
    assert gated(plan, ctypes.byref(a), None) == EINVAL
    assert gated(None, ctypes.byref(a), None) == EINVAL and gated(plan, None, None) == EINVAL
    lib.cleave_plan_destroy(plan)


def test_gated_8_bit_operands():
    plan = gated_plan(300, 200, 512, E4M3)
    for change in (dict(A=P + 8), dict(B_gate=P + 8), dict(B_up=P + 4), dict(lda=520), dict(ldb=520), dict(ldb=2 ** 22), dict(transB=0),
                   dict(dtype=BF16)):
        a = Args(A=P, B_gate=2 * P, B_up=3 * P, C=4 * P, scale_a=P, scale_gate=P, scale_up=P, lda=512, ldb=512, ldc=200, transB=1,
                 dtype=E4M3, out_dtype=BF16)
        for name, value in change.items():
            setattr(a, name, value)
        assert gated(plan, ctypes.byref(a), None) == EINVAL
    lib.cleave_plan_destroy(plan)


def test_gated_without_a_workspace():
    for dtype, change in ((F32, {}), (BF16, dict(lda=513)), (BF16, dict(ldb=516)), (BF16, dict(B_up=3 * P + 8)), (BF16, dict(A=P + 2)),
                          (BF16, dict(ldb=2 ** 21))):
        plan = gated_plan(300, 200, 512, dtype)
        a = Args(A=P, B_gate=2 * P, B_up=3 * P, C=4 * P, lda=512, ldb=512, ldc=200, transB=1, dtype=dtype, out_dtype=BF16)
        for name, value in change.items():
            setattr(a, name, value)
        assert gated(plan, ctypes.byref(a), None) == EINVAL
        lib.cleave_plan_destroy(plan)


@pytest.mark.parametrize("change", [
    dict(A=None), dict(B=None), dict(gate=None), dict(up=None), dict(dgate=None), dict(dup=None), dict(lda=511), dict(ldb=511),
    dict(ld_gate=199), dict(ld_up=199), dict(ld_dgate=199), dict(ld_dup=199), dict(transB=2), dict(dtype=E4M3), dict(out_dtype=E4M3),
    dict(act=4), dict(gate=P + 1), dict(dup=P + 1), dict(partials=P + 2), dict(dup=5 * P), dict(dgate=4 * P), dict(dup=3 * P),
    dict(dgate=3 * P, ld_dgate=208), dict(dup=4 * P, ld_up=208), dict(A=P + 2, partials=None), dict(dgate=P), dict(dup=2 * P)])
def test_grad(change):
    plan = made(300, 200, 512, BF16)
    a = GradArgs(A=P, B=2 * P, gate=3 * P, up=4 * P, dgate=5 * P, dup=6 * P, partials=7 * P, lda=512, ldb=512, ld_gate=200, ld_up=200,
                 ld_dgate=200, ld_dup=200, transB=1, dtype=BF16, out_dtype=BF16, act=3)
    for name, value in change.items():
        setattr(a, name, value)
    assert grad(plan, ctypes.byref(a), None) == EINVAL
    assert grad(None, ctypes.byref(a), None) == EINVAL and grad(plan, None, None) == EINVAL
    lib.cleave_plan_destroy(plan)


def test_plans_of_other_calls():
    for plan, call, args in ((made(300, 200, 512, BF16), gated, Args), (gated_plan(300, 200, 512, BF16), grad, GradArgs),
                             (made(300, 200, 512, E4M3), grad, GradArgs)):
        a = args(A=P, lda=512, ldb=512, transB=1, dtype=BF16, out_dtype=BF16)
        for name, kind in args._fields_:
            if kind is p and "scale" not in name:
                setattr(a, name, P * (1 + [n for n, _ in args._fields_].index(name)))
            elif name.startswith("ld") and name not in ("lda", "ldb"):
                setattr(a, name, 200)
        assert call(plan, ctypes.byref(a), None) == EINVAL
        lib.cleave_plan_destroy(plan)


@pytest.mark.parametrize("M", [4, 40, 900])
def test_plans_of_another_type(M):
    for plan_dtype, dtype in ((BF16, F32), (F32, BF16)):
        plan = gated_plan(M, 200, 512, plan_dtype)
        a = Args(A=P, B_gate=2 * P, B_up=3 * P, C=4 * P, partials=5 * P, lda=512, ldb=512, ldc=200, transB=1, dtype=dtype, out_dtype=BF16)
        assert gated(plan, ctypes.byref(a), None) == EINVAL
        lib.cleave_plan_destroy(plan)
        plan = made(M, 200, 512, plan_dtype)
        a = GradArgs(A=P, B=2 * P, gate=3 * P, up=4 * P, dgate=5 * P, dup=6 * P, partials=7 * P, lda=512, ldb=512, ld_gate=200, ld_up=200,
                     ld_dgate=200, ld_dup=200, transB=1, dtype=dtype, out_dtype=BF16)
        assert grad(plan, ctypes.byref(a), None) == EINVAL
        lib.cleave_plan_destroy(plan)


def test_other_calls_of_a_gated_plan_of_8_bit_operands():
    plan = gated_plan(300, 200, 512, E4M3)
    lists = ctypes.cast((p * 2)(P, 2 * P), p)
    execute = declare("cleave_execute_grouped", [p, p, i64, i64, p, i64, c_int, p, i64, c_int, c_int, p, p])
    reduce = declare("cleave_reduce_grouped", [p, p, i64, p, i64, c_int, p])
    assert execute(plan, None, 0, 2, lists, 512, 0, lists, 512, 1, BF16, P, None) == EINVAL
    assert reduce(plan, P, 2, lists, 200, F32, None) == EINVAL
    lib.cleave_plan_destroy(plan)


@pytest.mark.parametrize("M,N,K,dtype", [(300, 200, 512, F32), (2, 256, 8192, BF16), (300, 200, 513, BF16), (900, 200, 513, BF16)])
@pytest.mark.parametrize("change", [dict(partials=n * P) for n in range(1, 9)])
def test_a_workspace_in_another_ones_place(M, N, K, dtype, change):
    """Through partial blocks, few rows' sums, operands laid out again."""
    plan = gated_plan(M, N, K, dtype)
    a = Args(A=P, B_gate=2 * P, B_up=3 * P, C=4 * P, gate=5 * P, up=6 * P, bias_gate=7 * P, bias_up=8 * P, partials=9 * P, lda=K, ldb=K,
             ldc=N, ld_gate=N, ld_up=N, transB=1, dtype=dtype, out_dtype=BF16, act=3)
    for name, value in change.items():
        setattr(a, name, value)
    assert gated(plan, ctypes.byref(a), None) == EINVAL
    lib.cleave_plan_destroy(plan)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("change", [{out: n * P} for out in ("C", "gate", "up") for n in (7, 8, 10, 11, 12)])
def test_outputs_in_a_vectors_place(dtype, change):
    plan = gated_plan(300, 200, 512, dtype)
    a = Args(A=P, B_gate=2 * P, B_up=3 * P, C=4 * P, gate=5 * P, up=6 * P, bias_gate=7 * P, bias_up=8 * P, lda=512, ldb=512, ldc=200,
             ld_gate=200, ld_up=200, transB=1, dtype=dtype, out_dtype=BF16, act=3)
    if dtype == E4M3:
        a.scale_a, a.scale_gate, a.scale_up = 10 * P, 11 * P, 12 * P
    for name, value in change.items():
        setattr(a, name, value)
    if dtype == E4M3 or list(change.values())[0] < 10 * P:
        assert gated(plan, ctypes.byref(a), None) == EINVAL
    lib.cleave_plan_destroy(plan)


@pytest.mark.parametrize("M,K,dtype", [(300, 512, F32), (4, 512, BF16), (300, 513, BF16), (900, 513, BF16)])
@pytest.mark.parametrize("change", [dict(partials=n * P) for n in range(1, 7)])
def test_a_gradients_workspace_in_another_ones_place(M, K, dtype, change):
    plan = made(M, 200, K, dtype)
    a = GradArgs(A=P, B=2 * P, gate=3 * P, up=4 * P, dgate=5 * P, dup=6 * P, partials=7 * P, lda=K, ldb=K, ld_gate=200, ld_up=200,
                 ld_dgate=200, ld_dup=200, transB=1, dtype=dtype, out_dtype=BF16, act=3)
    for name, value in change.items():
        setattr(a, name, value)
    assert grad(plan, ctypes.byref(a), None) == EINVAL
    lib.cleave_plan_destroy(plan)
