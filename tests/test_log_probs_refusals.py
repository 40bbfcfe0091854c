"""What the C entry points of the log probabilities refuse, before anything is enqueued (the pointers are never followed)."""
import math

import pytest

from test_operator_refusals import BF16, E4M3, EINVAL, F32, OK, P, c_int, call, declare, f32, i64, p

ELIMIT = -4
log_probs = declare("cleave_log_probs", [i64, i64, p, i64, c_int, f32, p, p, p, p, i64, p, p, p, p])
workspace = declare("cleave_log_probs_workspace", [i64, i64, i64], i64)
backward = declare("cleave_log_probs_backward", [i64, i64, p, i64, c_int, f32, p, p, p, p, p, p, i64, p])

CALL = dict(rows=0, cols=100, x=P, ld=100, dtype=BF16, scale=1.0, ids=2 * P, logp=3 * P, lse=4 * P, ent=5 * P, n=20, top=6 * P, tl=7 * P,
            ws=None, stream=None)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(cols=0), dict(rows=2 ** 31), dict(cols=2 ** 30 + 1, ld=2 ** 31), dict(x=None), dict(ld=99), dict(dtype=E4M3),
    dict(dtype=5), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(ids=None), dict(logp=None),
    dict(n=-1), dict(n=0), dict(top=None), dict(tl=None), dict(n=20, cols=19), dict(x=P + 1), dict(ids=P + 4), dict(top=P + 4),
    dict(logp=P + 2), dict(lse=P + 2), dict(ent=P + 1), dict(tl=P + 2), dict(ws=P + 2), dict(dtype=F32, x=P + 2), dict(lse=3 * P),
    dict(ent=3 * P), dict(tl=3 * P), dict(ent=4 * P), dict(tl=4 * P), dict(tl=5 * P), dict(top=2 * P)])
def test_log_probs(change):
    assert call(log_probs, CALL) == OK
    assert call(log_probs, CALL, ids=None, logp=None, lse=None, ent=None, n=0, top=None, tl=None) == OK
    assert call(log_probs, CALL, **change) == EINVAL


def test_limit_and_workspace():
    assert call(log_probs, CALL, n=33) == ELIMIT and call(log_probs, CALL, n=32) == OK
    assert workspace(4, 100, 33) == ELIMIT and workspace(4, 100, 101) == EINVAL and workspace(4, 0, 0) == EINVAL
    assert workspace(-1, 100, 0) == EINVAL and workspace(4, 100, -1) == EINVAL and workspace(4, 2 ** 30 + 1, 0) == EINVAL
    assert workspace(1, 32000, 20) == 0 and workspace(4096, 250000, 20) == 0
    assert workspace(1, 250000, 20) > 0
    assert call(log_probs, CALL, rows=1, cols=250000, ld=250000) == EINVAL       # it is missing


BACKWARD = dict(rows=0, cols=100, x=P, ld=100, dtype=BF16, scale=1.0, ids=2 * P, lse=3 * P, dlogp=4 * P, ent=5 * P, dent=6 * P, dx=7 * P,
                ldd=100, stream=None)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(cols=0), dict(cols=2 ** 30 + 1, ld=2 ** 31, ldd=2 ** 31), dict(x=None), dict(lse=None), dict(dx=None), dict(ld=99),
    dict(ldd=99), dict(dtype=E4M3), dict(scale=0.0), dict(scale=math.nan), dict(ids=None), dict(dlogp=None), dict(ent=None), dict(dent=None),
    dict(ids=None, dlogp=None, ent=None, dent=None), dict(ids=P + 4), dict(lse=P + 2), dict(dx=P + 1), dict(dent=P + 2)])
def test_backward(change):
    assert call(backward, BACKWARD) == OK
    assert call(backward, BACKWARD, ids=None, dlogp=None) == OK and call(backward, BACKWARD, ent=None, dent=None) == OK
    assert call(backward, BACKWARD, dx=P) == OK
    assert call(backward, BACKWARD, **change) == EINVAL


def test_in_place_with_another_stride():
    assert call(backward, BACKWARD, rows=5, dx=P, ldd=104) == EINVAL


@pytest.mark.parametrize("change", [
    dict(logp=P), dict(lse=P), dict(ent=P), dict(tl=P), dict(top=P), dict(logp=2 * P), dict(lse=2 * P), dict(ent=2 * P), dict(tl=2 * P),
    dict(lse=6 * P), dict(ent=6 * P), dict(logp=6 * P), dict(tl=6 * P)])
def test_outputs_in_an_inputs_or_another_ones_place(change):
    assert call(log_probs, CALL, rows=5, **change) == EINVAL


@pytest.mark.parametrize("change", [dict(ws=n * P) for n in range(1, 8)])
def test_a_workspace_in_another_ones_place(change):
    """Where rows are taken in parts, every row's records are read while other rows' outputs are written."""
    assert call(log_probs, CALL, rows=2, cols=250000, ld=250000, **change) == EINVAL


@pytest.mark.parametrize("change", [dict(dx=n * P) for n in (2, 3, 4, 5, 6)])
def test_a_gradient_in_an_inputs_place(change):
    assert call(backward, BACKWARD, rows=5, **change) == EINVAL


def test_a_scale_whose_product_with_log_2_of_e_overflows():
    """(times a distance of zero, that of the largest logit, it would be NaN)"""
    for call_of, base in ((log_probs, CALL), (backward, BACKWARD)):
        assert call(call_of, base, scale=2.0 ** 127) == OK
        for scale in (2.0 ** 127 * (1 + 2.0 ** -23), 2.4e38, 3.4e38):
            assert call(call_of, base, scale=scale) == EINVAL
