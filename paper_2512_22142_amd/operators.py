"""Operators around the GEMMs of a layer's step: norm, linear product, bias gradient, AdamW.

Arguments are torch tensors on the current device, outputs and workspaces
included: nothing is allocated here.  `stream` is torch's current stream unless
one is given.  What each call computes and refuses is written in include/cleave.h.
"""
import ctypes

from . import _native
from .binding import BF16, F32, Plan, _check, _lib, _plan_addr

E4M3 = 2
ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "gelu_tanh": 2, "silu": 3}

_MOST = 2 ** 31 - 1


def rms_norm(x, weight, y, residual=None, sum_out=None, inv_rms=None, scales=None, eps=1e-5, stream=None):
    """cleave_rms_norm: y = h / rms(h) * weight for the rows of h = x + residual (x, residual, sum_out:
    fp32 or bf16; weight: fp32).  y has x's dtype, or float8_e4m3fn with one fp32 scale per row in
    `scales`.  sum_out gets h and inv_rms 1 / rms, which the gradient needs."""
    _check(_native.rms_norm(x, weight, y, residual, sum_out, inv_rms, scales, eps, stream), "cleave_rms_norm")


def _sizes(rows, cols):
    if not (0 <= rows <= _MOST and 1 <= cols <= _MOST):
        raise ValueError("rows x cols = %d x %d" % (rows, cols))
    return rows, cols


def rms_norm_workspace(rows, cols):
    """fp32 elements of rms_norm_backward's workspace."""
    return int(_lib.cleave_rms_norm_workspace(*_sizes(rows, cols)))


def rms_norm_backward(dy, h, weight, inv_rms, dx, dweight, workspace, dsum=None, stream=None):
    """cleave_rms_norm_backward: dx (the gradient of x and of the residual) and dweight from dy, the h and
    inv_rms that rms_norm left, and dsum, the gradient that reaches h through the residual stream."""
    _check(_native.rms_norm_backward(dy, h, weight, inv_rms, dx, dweight, workspace, dsum, stream), "cleave_rms_norm_backward")


def bias_grad_workspace(rows, cols):
    """fp32 elements of bias_grad's workspace."""
    return int(_lib.cleave_bias_grad_workspace(*_sizes(rows, cols)))


def bias_grad(dy, dbias, workspace, stream=None):
    """cleave_bias_grad: dbias (fp32) = sum of dy's rows."""
    _check(_native.bias_grad(dy, dbias, workspace, stream), "cleave_bias_grad")


def adamw(w, grads, m, v, lr, beta1, beta2, eps, weight_decay, step, m_scales=None, v_scales=None, copies=None,
          grad_scale=None, stream=None):
    """cleave_adamw: one AdamW step on the lists of tensors w (fp32, in place), grads (fp32 or bf16), m and v
    (in place: fp32, or float8_e4m3fn with a scale per 256 elements in m_scales and v_scales, v being
    held as its square root).  copies: bf16 tensors that get the new weights.  grad_scale: a
    device tensor of one element that the gradients are multiplied by.  lr, step and the others are host values, also in
    a graph: a recorded call repeats its step."""
    _check(_native.adamw(w, grads, m, v, m_scales, v_scales, copies, grad_scale, lr, beta1, beta2, eps, weight_decay, step,
                         stream), "cleave_adamw")


def plan_linear(M, N, K, dtype):
    """cleave_plan_linear: a plan for linear() with op(A) of M x K, op(B) of K x N and operands of torch dtype
    `dtype` (float32, bfloat16 or float8_e4m3fn).  plan.linear_workspace: fp32 elements of
    linear()'s `partials` (0: none needed)."""
    import torch
    codes = {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}
    if dtype not in codes:
        raise TypeError("unsupported dtype %s" % dtype)
    out = ctypes.c_void_p()
    _check(_lib.cleave_plan_linear(M, N, K, codes[dtype], ctypes.byref(out)), "cleave_plan_linear")
    plan = Plan(out.value)
    plan.linear_K = K
    return plan


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError("unknown activation %r: one of %s" % (name, ", ".join(sorted(k for k in ACTIVATIONS if k))))
    return ACTIVATIONS[name]


def linear(plan, A, B, C, transA=0, transB=0, bias=None, act=None, act_grad=None, residual=None, preact=None, scale_a=None,
           scale_b=None, partials=None, stream=None):
    """cleave_linear: C = act(op(A) op(B) + bias) + residual, `preact` (if given) getting the value in front of the
    activation; or, with act_grad naming an activation, C = (op(A) op(B)) act_grad'(preact) + residual.
    Operands in float8_e4m3fn: A is M x K, B is N x K (transB=1), with fp32 scales of their rows."""
    if act_grad is not None and act is not None:
        raise ValueError("act and act_grad exclude each other")
    code = _activation(act if act_grad is None else act_grad)
    _check(_native.linear(_plan_addr(plan), plan.M, plan.N, plan.linear_K, plan.linear_workspace, A, B, C, transA, transB, bias,
                          code, 0 if act_grad is None else 1, residual, preact, scale_a, scale_b, partials, stream),
           "cleave_linear")
