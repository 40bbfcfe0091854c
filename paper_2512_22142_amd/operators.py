"""Operators around the GEMMs of a layer's step: norms, linear and gated products, bias gradient, log probabilities, AdamW.

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


def _workspace(elems, where):
    if elems < 0:
        _check(elems, where)
    return int(elems)


def rms_norm_workspace(rows, cols):
    """fp32 elements of rms_norm_backward's workspace."""
    return int(_lib.cleave_rms_norm_workspace(*_sizes(rows, cols)))


def rms_norm_backward(dy, h, weight, inv_rms, dx, dweight, workspace, dsum=None, stream=None):
    """cleave_rms_norm_backward: dx (the gradient of x and of the residual) and dweight from dy, the h and
    inv_rms that rms_norm left, and dsum, the gradient that reaches h through the residual stream."""
    _check(_native.rms_norm_backward(dy, h, weight, inv_rms, dx, dweight, workspace, dsum, stream), "cleave_rms_norm_backward")


def layer_norm(x, weight, y, bias=None, residual=None, sum_out=None, mean=None, inv_std=None, scales=None, eps=1e-5, stream=None):
    """cleave_layer_norm: y = (h - mean(h)) / std(h) * weight + bias for the rows of h = x + residual (x, residual,
    sum_out: fp32 or bf16; weight, bias: fp32).  y has x's dtype, or float8_e4m3fn with one fp32 scale per row in
    `scales`.  sum_out gets h, mean and inv_std (1 / std) what the gradient needs."""
    _check(_native.layer_norm(x, weight, y, bias, residual, sum_out, mean, inv_std, scales, eps, stream), "cleave_layer_norm")


def layer_norm_workspace(rows, cols):
    """fp32 elements of layer_norm_backward's workspace."""
    return int(_lib.cleave_layer_norm_workspace(*_sizes(rows, cols)))


def layer_norm_backward(dy, h, weight, mean, inv_std, dx, dweight, workspace, dbias=None, dsum=None, stream=None):
    """cleave_layer_norm_backward: dx (the gradient of x and of the residual), dweight and dbias from dy, the h, mean and
    inv_std that layer_norm left, and dsum, the gradient that reaches h through the residual stream."""
    _check(_native.layer_norm_backward(dy, h, weight, mean, inv_std, dx, dweight, workspace, dbias, dsum, stream),
           "cleave_layer_norm_backward")


def bias_grad_workspace(rows, cols):
    """fp32 elements of bias_grad's workspace."""
    return int(_lib.cleave_bias_grad_workspace(*_sizes(rows, cols)))


def bias_grad(dy, dbias, workspace, stream=None):
    """cleave_bias_grad: dbias (fp32) = sum of dy's rows."""
    _check(_native.bias_grad(dy, dbias, workspace, stream), "cleave_bias_grad")


def log_probs_workspace(rows, cols, top=0):
    """fp32 elements of log_probs()'s workspace (0: none needed)."""
    return _workspace(_lib.cleave_log_probs_workspace(*_sizes(rows, cols), top), "cleave_log_probs_workspace")


def log_probs(logits, ids=None, logp=None, lse=None, entropy=None, top_ids=None, top_logp=None, scale=1.0, workspace=None, stream=None):
    """cleave_log_probs: for the rows of scale * logits (fp32 or bf16) the log probability of each row's token in ids (int64; negative:
    no token, 0), the log of the sum of exponentials, the entropy, and the most likely tokens in descending order, as many
    as top_ids (int64) and top_logp have columns.  The other outputs are fp32, one element per row; what is None is left out."""
    _check(_native.log_probs(logits, ids, logp, lse, entropy, top_ids, top_logp, scale, workspace, stream), "cleave_log_probs")


def log_probs_backward(logits, lse, dlogits, ids=None, dlogp=None, entropy=None, dentropy=None, scale=1.0, stream=None):
    """cleave_log_probs_backward: dlogits (the logits' dtype; may be the logits themselves) from the gradients dlogp of the tokens'
    log probabilities and dentropy of the entropy, with the lse and entropy that log_probs left."""
    _check(_native.log_probs_backward(logits, lse, dlogits, ids, dlogp, entropy, dentropy, scale, stream), "cleave_log_probs_backward")


def adamw(w, grads, m, v, lr, beta1, beta2, eps, weight_decay, step, m_scales=None, v_scales=None, copies=None,
          grad_scale=None, stream=None):
    """cleave_adamw: one AdamW step on the lists of tensors w (fp32, in place), grads (fp32 or bf16), m and v
    (in place: fp32, or float8_e4m3fn with a scale per 256 elements in m_scales and v_scales, v being
    held as its square root).  copies: bf16 tensors that get the new weights.  grad_scale: a
    device tensor of one element that the gradients are multiplied by.  lr, step and the others are host values, also in
    a graph: a recorded call repeats its step."""
    _check(_native.adamw(w, grads, m, v, m_scales, v_scales, copies, grad_scale, lr, beta1, beta2, eps, weight_decay, step,
                         stream), "cleave_adamw")


def _operand_code(dtype):
    import torch
    codes = {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}
    if dtype not in codes:
        raise TypeError("unsupported dtype %s" % dtype)
    return codes[dtype]


def plan_linear(M, N, K, dtype):
    """cleave_plan_linear: a plan for linear() with op(A) of M x K, op(B) of K x N and operands of torch dtype
    `dtype` (float32, bfloat16 or float8_e4m3fn).  plan.linear_workspace: fp32 elements of
    linear()'s `partials` (0: none needed)."""
    out = ctypes.c_void_p()
    _check(_lib.cleave_plan_linear(M, N, K, _operand_code(dtype), ctypes.byref(out)), "cleave_plan_linear")
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


def plan_gated(M, N, K, dtype):
    """cleave_plan_gated: a plan for linear_gated() with A of M x K, both weights of K x N and operands of torch dtype
    `dtype` (float32, bfloat16 or float8_e4m3fn)."""
    out = ctypes.c_void_p()
    _check(_lib.cleave_plan_gated(M, N, K, _operand_code(dtype), ctypes.byref(out)), "cleave_plan_gated")
    plan = Plan(out.value)
    plan.linear_K = K
    return plan


def gated_workspace(plan, whole=False):
    """fp32 elements of linear_gated()'s `partials` (0: none needed).  whole=True: for bf16 operands that start on 16 bytes, with
    row strides and K (and, with transB=0, N) in multiples of 8."""
    return _workspace(_lib.cleave_gated_workspace(plan._h, int(bool(whole))), "cleave_gated_workspace")


def linear_gated(plan, A, B_gate, B_up, C, transB=0, act="silu", bias_gate=None, bias_up=None, gate=None, up=None, scale_a=None,
                 scale_gate=None, scale_up=None, partials=None, stream=None):
    """cleave_linear_gated: C = act(A op(B_gate) + bias_gate) * (A op(B_up) + bias_up); `gate` and `up` (if given) get the
    two factors' sums, which the gradient needs.  B_gate and B_up share their row stride.  Operands in float8_e4m3fn: both
    weights N x K (transB=1), with fp32 scales of the rows of A and of the weights."""
    _check(_native.linear_gated(_plan_addr(plan), plan.M, plan.N, plan.linear_K, A, B_gate, B_up, C, transB, _activation(act),
                                bias_gate, bias_up, gate, up, scale_a, scale_gate, scale_up, partials, stream), "cleave_linear_gated")


def gated_grad_workspace(plan, whole=False):
    """fp32 elements of linear_gated_grad()'s `partials` (0: none needed) with plan_linear's plan; whole as for gated_workspace."""
    return _workspace(_lib.cleave_gated_grad_workspace(plan._h, int(bool(whole))), "cleave_gated_grad_workspace")


def linear_gated_grad(plan, A, B, gate, up, dgate, dup, transB=0, act="silu", partials=None, stream=None):
    """cleave_linear_gated_grad: with p = A op(B), the gradient behind the gated product, dgate = p * up * act'(gate) and
    dup = p * act(gate) from the gate and up that linear_gated kept.  plan: plan_linear's of that product."""
    _check(_native.linear_gated_grad(_plan_addr(plan), plan.M, plan.N, plan.linear_K, A, B, gate, up, dgate, dup, transB,
                                     _activation(act), partials, stream), "cleave_linear_gated_grad")
