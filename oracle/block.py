"""CPU oracle for the transformer-block operators, in 64 bits from their formulas, with bounds on what a computation may be off.

TEST INFRASTRUCTURE ONLY.  Never imported by the product path.

    gated   [G U] = X Win,  H = act(G) * U,  Y = H Wout + R
            dH = dY Wout^T,  dG = dH * U * act'(G),  dU = dH * act(G),  dX = [dG dU] Win^T,  dWin = X^T [dG dU],  dWout = H^T dY
    dense   Z = X W + b,  Y = act(Z) + R;  dZ = dY * act'(Z),  dX = dZ W^T,  dW = X^T dZ,  db = column sums of dZ
    clip    norm = sqrt(sum g^2),  c = min(1, max_norm / norm),  g <- c g;  wm <- wm - lr (c g),  wb <- wm

Every result is a pair (value, bound).  The bounds follow the definition of the calls: products of bf16 numbers are exact in
float, a float sum of n terms is off by at most (n + 2) 2^-24 times the sum of their magnitudes, and what is rounded to bf16 for a
second product (H, [dG dU], dZ) by half a step, 2^-8 of it; an error of a factor goes through a product with the magnitudes
of the other.  Activations in kernels that round to bf16 may be off by 1e-6 of |z| (their polynomial and the hardware's
exponential), slopes by 3e-5; where the result stays float, activations by 4 steps of 2^-24.
"""
import numpy as np
from scipy.special import erfc

NONE, RELU, GELU, SILU = 0, 1, 2, 3
STEP, HALF = 2.0 ** -24, 2.0 ** -8          # half steps of float and bf16
SLOPE_MAX, CURVE_MAX = 1.13, 0.81            # largest |act'| and |act''| of all of them (away from ReLU's corner)


def act(z, kind):
    if kind == RELU:
        return np.where(z < 0, 0.0, z)
    if kind == GELU:
        return 0.5 * z * erfc(-z / np.sqrt(2))
    if kind == SILU:
        return z / (1 + np.exp(-z))
    return z


def slope(z, kind):
    if kind == RELU:
        return np.where(np.isnan(z), z, (z > 0).astype(np.float64))
    if kind == GELU:
        return 0.5 * erfc(-z / np.sqrt(2)) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if kind == SILU:
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def product(a, b, ea=None, eb=None):
    """(a b, bound); ea, eb: bounds of the factors."""
    v, size = a @ b, np.abs(a) @ np.abs(b)
    e = (a.shape[1] + 2) * STEP * size
    if ea is not None:
        e = e + ea @ np.abs(b)
    if eb is not None:
        e = e + np.abs(a) @ eb + (0 if ea is None else ea @ eb)
    return v, e


def rounded(v, e, bf16=True):
    return v, e + (HALF if bf16 else STEP) * (np.abs(v) + e)


def activated(z, ez, kind, fine=False):
    a = act(z, kind)
    own = 0.0 if kind in (NONE, RELU) else 4 * STEP * np.abs(a) + 4 * STEP * np.abs(z) if fine else 1e-6 * np.abs(z) + 4e-7
    return a, SLOPE_MAX * ez + own


def gated_forward(x, w_in, w_out, r, kind):
    """Returns dict(gu, h, y) of (value, bound)."""
    F = w_out.shape[0]
    gu, egu = product(x, w_in)
    a, ea = activated(gu[:, :F], egu[:, :F], kind)
    u, eu = gu[:, F:], egu[:, F:]
    h, eh = rounded(a * u, ea * np.abs(u) + np.abs(a) * eu + ea * eu)
    y, ey = product(h, w_out, eh)
    if r is not None:
        y, ey = y + r, ey + STEP * (np.abs(y) + np.abs(r))
    return dict(gu=rounded(gu, egu, False), h=(h, eh), y=rounded(y, ey))


def gated_backward(x, w_in, w_out, h, gu, dy, kind, fine=False):
    """From what the forward pass left in h (bf16) and gu (float).  fine: slopes within what dense_backward allows, 8 steps of 2^-24 (1 + |z|)."""
    F = w_out.shape[0]
    g, u = gu[:, :F], gu[:, F:]
    dh, edh = product(dy, w_out.T)
    a, ea = activated(g, 0.0, kind)
    d = slope(g, kind)
    ed = np.zeros_like(d) if kind in (NONE, RELU) else 8 * STEP * (1 + np.abs(g)) if fine else np.full_like(d, 3e-5)
    dg = dh * u * d
    edg = edh * np.abs(u * d) + np.abs(dh * u) * ed + edh * np.abs(u) * ed + 3 * STEP * np.abs(dg)
    du = dh * a
    edu = edh * np.abs(a) + np.abs(dh) * ea + edh * ea + STEP * np.abs(du)
    dgu, edgu = rounded(np.concatenate([dg, du], 1), np.concatenate([edg, edu], 1))
    return dict(dx=rounded(*product(dgu, w_in.T, edgu)), dw_in=rounded(*product(x.T, dgu, None, edgu)), dw_out=rounded(*product(h.T, dy)))


def dense_forward(x, w, b, r, kind, bf16):
    z, ez = product(x, w)
    if b is not None:
        z = z + b
        ez = ez + STEP * np.abs(z)
    y, ey = activated(z, ez, kind, not bf16)
    if r is not None:
        y = y + r
        ey = ey + STEP * np.abs(y)
    return dict(z=rounded(z, ez, False), y=rounded(y, ey, bf16))


def dense_backward(x, w, z, dy, kind):
    """From what the forward pass left in z (float; not used without an activation)."""
    if kind == NONE:
        dz, edz = dy, np.zeros_like(dy)
        rz, erz = dz, edz
    else:
        d = slope(z, kind)
        dz = dy * d
        edz = np.abs(dy) * (0.0 if kind == RELU else 8 * STEP * (1 + np.abs(z))) + STEP * np.abs(dz)
        rz, erz = rounded(dz, edz)
    M = x.shape[0]
    db, edb = dz.sum(0), edz.sum(0) + (M + 2) * STEP * np.abs(dz).sum(0)
    return dict(dx=rounded(*product(rz, w.T, erz)), dw=rounded(*product(x.T, rz, None, erz)), db=(db, edb))


def clip(tensors, max_norm):
    """tensors: float64 arrays.  Returns (norm, coefficient)."""
    norm = np.sqrt(sum(float((t * t).sum()) for t in tensors))
    with np.errstate(divide="ignore", invalid="ignore"):
        ratio = np.float64(1) if norm <= max_norm else np.float64(max_norm) / np.float64(norm)
    return norm, ratio if ratio < 1 or np.isnan(ratio) else 1.0
