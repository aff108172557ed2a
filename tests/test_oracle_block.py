"""Pins of the block oracle: values against torch in double, gradients against torch's and against central differences."""
import numpy as np
import pytest
import torch

from oracle import block

TORCH = {block.NONE: lambda z: z, block.RELU: torch.relu, block.GELU: torch.nn.functional.gelu, block.SILU: torch.nn.functional.silu}


def close(a, b, tol=1e-12):
    assert np.abs(a - b).max() <= tol * max(1.0, np.abs(b).max())


@pytest.mark.parametrize("kind", list(TORCH))
def test_activations_and_slopes(kind):
    z = torch.linspace(-9, 9, 4001, dtype=torch.float64).requires_grad_()
    a = TORCH[kind](z)
    a.sum().backward()
    close(block.act(z.detach().numpy(), kind), a.detach().numpy())
    away = np.abs(z.detach().numpy()) > 1e-9
    close(block.slope(z.detach().numpy(), kind)[away], z.grad.numpy()[away])
    assert np.abs(block.slope(z.detach().numpy(), kind)).max() <= block.SLOPE_MAX


@pytest.mark.parametrize("kind", list(TORCH))
def test_gated_block_and_gradients(kind):
    rng = np.random.default_rng(kind)
    M, K, F, N = 5, 7, 6, 4
    x, w_in, w_out, r, dy = (rng.standard_normal(s) for s in ((M, K), (K, 2 * F), (F, N), (M, N), (M, N)))
    t = [torch.tensor(v, requires_grad=True) for v in (x, w_in, w_out)]
    gu = t[0] @ t[1]
    y = (TORCH[kind](gu[:, :F]) * gu[:, F:]) @ t[2] + torch.tensor(r)
    y.backward(torch.tensor(dy))
    f = block.gated_forward(x, w_in, w_out, r, kind)
    close(f["y"][0], y.detach().numpy())
    b = block.gated_backward(x, w_in, w_out, f["h"][0], f["gu"][0], dy, kind)
    for name, grad in zip(("dx", "dw_in", "dw_out"), t):
        close(b[name][0], grad.grad.numpy())
    # differences, along one direction of every input
    for i, name in enumerate(("dx", "dw_in", "dw_out")):
        d = rng.standard_normal((x, w_in, w_out)[i].shape)
        at = lambda s: (block.gated_forward(*[v + s * d if j == i else v for j, v in enumerate((x, w_in, w_out))], r, kind)["y"][0] * dy).sum()
        assert abs((at(1e-6) - at(-1e-6)) / 2e-6 - (b[name][0] * d).sum()) < 1e-5 * max(1, abs((b[name][0] * d).sum()))


@pytest.mark.parametrize("kind", list(TORCH))
def test_dense_layer_and_gradients(kind):
    rng = np.random.default_rng(10 + kind)
    M, K, N = 6, 5, 4
    x, w, bias, r, dy = (rng.standard_normal(s) for s in ((M, K), (K, N), (N,), (M, N), (M, N)))
    t = [torch.tensor(v, requires_grad=True) for v in (x, w, bias)]
    y = TORCH[kind](t[0] @ t[1] + t[2]) + torch.tensor(r)
    y.backward(torch.tensor(dy))
    f = block.dense_forward(x, w, bias, r, kind, True)
    close(f["y"][0], y.detach().numpy())
    b = block.dense_backward(x, w, f["z"][0], dy, kind)
    for name, grad in zip(("dx", "dw", "db"), t):
        close(b[name][0], grad.grad.numpy())
    for i, name in enumerate(("dx", "dw", "db")):
        d = rng.standard_normal((x, w, bias)[i].shape)
        at = lambda s: (block.dense_forward(*[v + s * d if j == i else v for j, v in enumerate((x, w, bias))], r, kind, True)["y"][0] * dy).sum()
        assert abs((at(1e-6) - at(-1e-6)) / 2e-6 - (b[name][0] * d).sum()) < 1e-5 * max(1, abs((b[name][0] * d).sum()))


def test_clip():
    t = [np.array([3.0, 0.0]), np.array([[4.0]])]
    assert block.clip(t, 1.0) == (5.0, 0.2)
    assert block.clip(t, 5.0) == (5.0, 1.0)
    assert block.clip(t, 10.0) == (5.0, 1.0)
    assert block.clip([np.zeros(3)], 1.0) == (0.0, 1.0)
    assert block.clip(t, np.inf) == (5.0, 1.0)
    assert np.isnan(block.clip([np.array([np.nan, 1.0])], 1.0)[1])
    assert block.clip([np.array([np.inf, 1.0])], 1.0) == (np.inf, 0.0)


def test_the_bounds_notice_a_mistake():
    """A residual left out, a bias twice, halves exchanged: far outside what rounding allows (the mistake is in the oracle's call)."""
    rng = np.random.default_rng(3)
    x, w_in, w_out, r = (rng.standard_normal(s) for s in ((9, 24), (24, 32), (16, 8), (9, 8)))
    w_in /= np.sqrt(24)
    w_out /= 4
    v, e = block.gated_forward(x, w_in, w_out, r, block.SILU)["y"]
    swapped = np.concatenate([w_in[:, 16:], w_in[:, :16]], 1)
    for wrong in (block.gated_forward(x, w_in, w_out, None, block.SILU), block.gated_forward(x, swapped, w_out, r, block.SILU),
                  block.gated_forward(x, w_in, w_out, r, block.GELU)):
        assert (np.abs(wrong["y"][0] - v) > e).mean() > 0.2
