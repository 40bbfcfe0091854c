"""Oracle of the operators around the GEMMs, in fp64 numpy, from their formulas.

Shares no code with the library.  Values that the library holds in 8 bits come in and
go out as the numbers they stand for.
"""
import math

import numpy as np

E4M3_MAX = 448.0
LEAST = 2.0 ** -100
STATE_BLOCK = 256


def round_e4m3(x):
    """Nearest e4m3 value, ties to the even mantissa (|x| up to 448 and a little)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    with np.errstate(divide="ignore"):
        e = np.where(a > 0, np.floor(np.log2(np.where(a > 0, a, 1.0))), -6.0)
    step = 2.0 ** (np.maximum(e, -6.0) - 3)
    return np.copysign(np.minimum(np.rint(a / step) * step, E4M3_MAX), x)


def rms_norm(x, w, eps, residual=None):
    """(y, h, 1 / rms) of the rows of h = x + residual."""
    h = x if residual is None else x + residual
    inv = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return h * inv[:, None] * w, h, inv


def row_scales(y):
    most = np.abs(y).max(axis=1)
    return np.where(most < LEAST, 0.0, most / E4M3_MAX)


def rms_norm_backward(dy, h, w, inv, dsum=None):
    """(dx, dw) with the given 1 / rms."""
    xhat = h * inv[:, None]
    g = dy * w
    dx = inv[:, None] * (g - xhat * (g * xhat).mean(axis=1, keepdims=True))
    if dsum is not None:
        dx = dx + dsum
    return dx, (dy * xhat).sum(axis=0)


_K = math.sqrt(2.0 / math.pi)


def act(z, name):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(_K * (z + 0.044715 * z ** 3)))
    return z


def act_grad(z, name):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "silu":
        p = 1.0 / (1.0 + np.exp(-z))
        return p + z * p * (1.0 - p)
    if name == "gelu_tanh":
        t = np.tanh(_K * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * _K * (1.0 + 3 * 0.044715 * z * z)
    return np.ones_like(z)


def linear(a, b, bias=None, name="none", residual=None, scale_a=None, scale_b=None):
    """(y, z): z = a . b (scales of a's rows and b's columns) + bias, y = act(z) + residual."""
    z = a @ b
    if scale_a is not None:
        z = z * scale_a[:, None] * scale_b
    if bias is not None:
        z = z + bias
    y = act(z, name)
    return (y if residual is None else y + residual), z


def adamw(w, g, m, v, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0):
    """(w, m, v) after one step."""
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    w = w - lr * ((m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps) + weight_decay * w)
    return w, m, v


def block_scales(x):
    """One scale for each 256 consecutive values."""
    blocks = -(-x.size // STATE_BLOCK)
    pad = np.zeros(blocks * STATE_BLOCK)
    pad[: x.size] = np.abs(x)
    most = pad.reshape(blocks, STATE_BLOCK).max(axis=1)
    return np.where(most < LEAST, 0.0, most / E4M3_MAX)
