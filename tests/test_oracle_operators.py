"""Pins of the oracle of the operators around the GEMMs (CPU)."""
import numpy as np
import pytest
import torch

from oracle import operators as oo


def _differences(f, x, step=1e-5):
    """Central differences of the scalar f at x, element by element."""
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + step
        up = f()
        x[i] = keep - step
        down = f()
        x[i] = keep
        out[i] = (up - down) / (2 * step)
    return out


def test_e4m3_rounding_is_torchs():
    x = np.concatenate([np.linspace(-448, 448, 40001), np.linspace(-0.05, 0.05, 20001), [2.0 ** -10, 2.0 ** -9, 0.0]])
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(oo.round_e4m3(x), want)


def test_norm_by_hand():
    y, h, inv = oo.rms_norm(np.array([[3.0, 4.0]]), np.array([2.0, 10.0]), 0.0)
    assert np.allclose(inv, np.sqrt(2) / 5) and np.allclose(y, [[6 * np.sqrt(2) / 5, 40 * np.sqrt(2) / 5]])
    y, h, _ = oo.rms_norm(np.array([[1.0, 1.0]]), np.ones(2), 0.0, residual=np.array([[1.0, 1.0]]))
    assert np.array_equal(h, [[2.0, 2.0]]) and np.allclose(y, 1.0)
    assert np.array_equal(oo.row_scales(np.array([[0.0, 0.0], [448.0, -896.0]])), [0.0, 2.0])


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(0)
    x, r, w = rng.normal(size=(3, 7)), rng.normal(size=(3, 7)), rng.normal(size=7)
    c, d = rng.normal(size=(3, 7)), rng.normal(size=(3, 7))

    def loss():   # the norm's output and the residual stream are both used
        y, h, _ = oo.rms_norm(x, w, 1e-3, r)
        return (c * y).sum() + (d * h).sum()

    _, h, inv = oo.rms_norm(x, w, 1e-3, r)
    dx, dw = oo.rms_norm_backward(c, h, w, inv, d)
    # (relative to 1: the second-order term of a step of 1e-5 is 1e-10, rounding 1e-16 / 1e-5)
    assert np.allclose(dx, _differences(loss, x), atol=1e-8)
    assert np.allclose(dx, _differences(loss, r), atol=1e-8)
    assert np.allclose(dw, _differences(loss, w), atol=1e-8)


@pytest.mark.parametrize("name", ["none", "silu", "gelu_tanh", "relu"])
def test_activation_gradients_against_differences(name):
    z = np.linspace(-6, 6, 101) + 0.013   # no value at relu's corner
    want = (oo.act(z + 1e-6, name) - oo.act(z - 1e-6, name)) / 2e-6
    assert np.allclose(oo.act_grad(z, name), want, atol=1e-8)
    if name in ("silu", "gelu_tanh"):
        lib = {"silu": torch.nn.functional.silu, "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[name]
        assert np.allclose(oo.act(z, name), lib(torch.from_numpy(z)).numpy(), atol=1e-14)


def test_linear_gradients_against_differences():
    rng = np.random.default_rng(1)
    z0, w, b, c = rng.normal(size=(4, 5)), rng.normal(size=(5, 3)), rng.normal(size=3), rng.normal(size=(4, 3))

    def loss():   # act(z0) . w + b, as an MLP's second product
        return (c * oo.linear(oo.act(z0, "gelu_tanh"), w, b)[0]).sum()

    assert np.allclose((c @ w.T) * oo.act_grad(z0, "gelu_tanh"), _differences(loss, z0), atol=1e-8)
    assert np.allclose(oo.act(z0, "gelu_tanh").T @ c, _differences(loss, w), atol=1e-8)
    assert np.allclose(c.sum(axis=0), _differences(loss, b), atol=1e-8)


def test_adamw_is_the_library_optimizers():
    rng = np.random.default_rng(2)
    w, m, v = rng.normal(size=50), np.zeros(50), np.zeros(50)
    p = torch.nn.Parameter(torch.from_numpy(w.copy()))
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    for step in range(1, 6):
        g = rng.normal(size=50)
        w, m, v = oo.adamw(w, 2 * g, m, v, 1e-2, 0.9, 0.95, 1e-8, 0.1, step, grad_scale=0.5)
        p.grad = torch.from_numpy(g)
        opt.step()
    # (the library decays before the update and not beside it: the same but for rounding)
    assert np.allclose(w, p.detach().numpy(), rtol=0, atol=1e-12)


def test_block_scales():
    x = np.zeros(257)
    x[3], x[256] = -896.0, 448.0
    assert np.array_equal(oo.block_scales(x), [2.0, 1.0])
    assert np.array_equal(oo.block_scales(np.full(3, 1e-31)), [0.0])
