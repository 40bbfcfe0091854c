"""What the C entry points of the layer norm refuse, before anything is enqueued (the pointers are never followed)."""
import math

import pytest

from test_operator_refusals import BF16, E4M3, EINVAL, F32, OK, P, c_int, call, declare, f32, i64, p

norm = declare("cleave_layer_norm", [i64, i64, p, i64, p, i64, c_int, p, p, f32, p, i64, c_int, p, p, i64, p, p, p])
backward = declare("cleave_layer_norm_backward", [i64, i64, p, i64, p, i64, p, i64, c_int, p, p, p, p, i64, p, p, p, p])
workspace = declare("cleave_layer_norm_workspace", [i64, i64], i64)

NORM = dict(rows=0, cols=100, x=P, ldx=100, r=2 * P, ldr=100, dtype=BF16, w=3 * P, b=4 * P, eps=1e-5, y=5 * P, ldy=100, y_dtype=BF16,
            scales=None, h=6 * P, ldh=100, mean=7 * P, inv=8 * P, stream=None)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(cols=0), dict(rows=2 ** 31), dict(cols=2 ** 31, ldx=2 ** 32, ldr=2 ** 32, ldy=2 ** 32, ldh=2 ** 32),
    dict(dtype=E4M3, y_dtype=E4M3, scales=P), dict(dtype=7, y_dtype=7), dict(y_dtype=F32), dict(y_dtype=E4M3), dict(scales=P),
    dict(x=None), dict(w=None), dict(y=None), dict(ldx=99), dict(ldr=99), dict(ldy=99), dict(ldh=99), dict(x=P + 1), dict(r=P + 1),
    dict(y=P + 1), dict(h=P + 1), dict(w=P + 2), dict(b=P + 2), dict(mean=P + 2), dict(inv=P + 2), dict(eps=-1e-6), dict(eps=math.inf),
    dict(eps=math.nan), dict(dtype=F32, y_dtype=F32, x=P + 2)])
def test_norm(change):
    assert call(norm, NORM) == OK
    assert call(norm, NORM, r=None, ldr=0, h=None, ldh=0, mean=None, inv=None, b=None) == OK
    assert call(norm, NORM, y_dtype=E4M3, scales=9 * P, y=5 * P + 1) == OK
    assert call(norm, NORM, **change) == EINVAL


@pytest.mark.parametrize("change", [
    dict(y_dtype=E4M3, scales=9 * P, y=P), dict(y_dtype=E4M3, scales=9 * P, y=2 * P), dict(y_dtype=E4M3, scales=9 * P, y=6 * P),
    dict(y=P, ldy=104), dict(y=2 * P, ldr=104), dict(h=P, ldx=101), dict(h=2 * P, ldh=200), dict(y=6 * P), dict(mean=8 * P)])
def test_shared_addresses(change):
    assert call(norm, NORM, **change) == OK       # no rows: nothing is read or written
    assert call(norm, NORM, **{"rows": 5, **change}) == EINVAL


BACKWARD = dict(rows=5, cols=100, dy=P, lddy=100, h=2 * P, ldh=100, ds=3 * P, ldds=100, dtype=BF16, w=4 * P, mean=5 * P, inv=6 * P,
                dx=7 * P, lddx=100, dw=8 * P, db=9 * P, ws=10 * P, stream=None)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(cols=0), dict(dtype=E4M3), dict(dy=None), dict(h=None), dict(w=None), dict(mean=None), dict(inv=None),
    dict(dx=None), dict(dw=None), dict(ws=None), dict(lddy=99), dict(ldh=99), dict(ldds=99), dict(lddx=99), dict(dy=P + 1),
    dict(ds=P + 1), dict(ws=P + 2), dict(db=P + 2), dict(mean=P + 2), dict(db=8 * P), dict(dx=P, lddx=104), dict(dx=2 * P, ldh=104),
    dict(dx=3 * P, ldds=101)])
def test_backward(change):
    assert call(backward, BACKWARD, **change) == EINVAL


def test_workspace():
    assert workspace(-1, 8) == EINVAL and workspace(8, 0) == EINVAL and workspace(2 ** 31, 8) == EINVAL and workspace(8, 2 ** 31) == EINVAL
    for rows, cols in ((0, 8), (1, 1), (5000, 4096), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert workspace(rows, cols) >= 2 * cols and workspace(rows, cols) % 8 == 0


@pytest.mark.parametrize("change", [
    dict(mean=9 * P), dict(inv=9 * P), dict(mean=3 * P), dict(inv=4 * P), dict(scales=3 * P), dict(scales=4 * P), dict(scales=5 * P),
    dict(scales=6 * P), dict(mean=5 * P), dict(mean=6 * P), dict(inv=P), dict(mean=2 * P), dict(y=3 * P), dict(h=4 * P)])
def test_rows_statistics_in_another_ones_place(change):
    """Scales, mean and inv_std are written row by row, while other rows are read and written."""
    eight = {**NORM, "y_dtype": E4M3, "scales": 9 * P, **change}
    assert call(norm, eight) == OK       # no rows
    assert call(norm, eight, rows=5) == EINVAL


@pytest.mark.parametrize("change", [
    dict(dw=10 * P), dict(db=10 * P), dict(dx=10 * P), dict(dx=8 * P), dict(dx=9 * P), dict(dx=4 * P), dict(dx=5 * P), dict(dx=6 * P),
    dict(ws=P), dict(ws=2 * P), dict(ws=3 * P), dict(ws=4 * P), dict(ws=5 * P), dict(ws=6 * P)])
def test_gradients_in_another_ones_place(change):
    assert call(backward, BACKWARD, **change) == EINVAL
