"""The operators of the transformer block around the layer -- TEST
INFRASTRUCTURE ONLY.

Sec. 4.1 ("Model Design") keeps Equiformer's graph transformer around the
tensor products: a norm, the attention block, a norm, a feed-forward block,
each under a skip connection.  The paper gives no equations for norm and
feed-forward block; this module fixes the reading that the GPU path implements,
in float64, with the gradients written out.

Layer norm, per node and degree l over 2l + 1 rows and C channels: xc = x less
its channel mean for l = 0, x otherwise; xhat = xc / sqrt(mean(xc^2) + eps);
y = gamma[l] xhat, plus beta for l = 0.

Gated feed-forward block: y = ((x w_up) * act(x[:, 0] w_gate + b_gate)) w_down
+ residual, the gate shared by a node's rows.
"""
from __future__ import annotations

import math

import numpy as np


def degrees(d: int):
    """(l, rows) of each degree of d = (L + 1)^2 rows."""
    return [(l, slice(l * l, (l + 1) ** 2)) for l in range(math.isqrt(d))]


def _normalised(x, l, eps):
    xc = x - x.mean(axis=2, keepdims=True) if l == 0 else x
    r = 1.0 / np.sqrt((xc * xc).mean(axis=(1, 2), keepdims=True) + eps)
    return xc * r, r


def layer_norm(x, gamma, beta, eps):
    x, gamma = np.asarray(x, np.float64), np.asarray(gamma, np.float64)
    y = np.empty_like(x)
    for l, rows in degrees(x.shape[1]):
        y[:, rows] = _normalised(x[:, rows], l, eps)[0] * gamma[l]
    if beta is not None:
        y[:, 0] += np.asarray(beta, np.float64)
    return y


def layer_norm_backward(x, gamma, grad_y, eps, grad_res=None):
    """(grad_x, grad_gamma, grad_beta)."""
    x, gamma, grad_y = (np.asarray(v, np.float64) for v in (x, gamma, grad_y))
    gx, gg = np.empty_like(x), np.empty_like(gamma)
    for l, rows in degrees(x.shape[1]):
        xhat, r = _normalised(x[:, rows], l, eps)
        w = grad_y[:, rows] * gamma[l]
        g = w - xhat * (w * xhat).mean(axis=(1, 2), keepdims=True)
        if l == 0:
            g = g - w.mean(axis=2, keepdims=True)
        gx[:, rows] = r * g
        gg[l] = (grad_y[:, rows] * xhat).sum(axis=(0, 1))
    if grad_res is not None:
        gx = gx + np.asarray(grad_res, np.float64)
    return gx, gg, grad_y[:, 0].sum(axis=0)


def _erf(v):
    from scipy.special import erf

    return erf(v)


def activation(q, act):
    """act(q) and its derivative."""
    if act == "gelu":
        cdf = 0.5 * (1.0 + _erf(q / math.sqrt(2.0)))
        return q * cdf, cdf + q * np.exp(-0.5 * q * q) / math.sqrt(2.0 * math.pi)
    sig = 1.0 / (1.0 + np.exp(-q))
    if act == "sigmoid":
        return sig, sig * (1.0 - sig)
    if act == "silu":
        return q * sig, sig + q * sig * (1.0 - sig)
    raise ValueError(act)


def gated_ffn(x, w_up, w_gate, w_down, b_gate=None, residual=None, act="silu"):
    x, w_up, w_gate, w_down = (np.asarray(v, np.float64) for v in (x, w_up, w_gate, w_down))
    q = x[:, 0] @ w_gate + (0.0 if b_gate is None else np.asarray(b_gate, np.float64))
    y = ((x @ w_up) * activation(q, act)[0][:, None]) @ w_down
    return y if residual is None else y + np.asarray(residual, np.float64)


def gated_ffn_backward(x, w_up, w_gate, w_down, grad_y, b_gate=None, act="silu"):
    """(grad_x, grad_w_up, grad_w_gate, grad_w_down, grad_b_gate)."""
    x, w_up, w_gate, w_down, gy = (np.asarray(v, np.float64) for v in (x, w_up, w_gate, w_down, grad_y))
    C, F = w_up.shape
    q = x[:, 0] @ w_gate + (0.0 if b_gate is None else np.asarray(b_gate, np.float64))
    s, ds = activation(q, act)
    u, dh = x @ w_up, gy @ w_down.T
    dq = (dh * u).sum(axis=1) * ds
    du, h = dh * s[:, None], u * s[:, None]
    gx = du @ w_up.T
    gx[:, 0] += dq @ w_gate.T
    return (gx, x.reshape(-1, C).T @ du.reshape(-1, F), x[:, 0].T @ dq, h.reshape(-1, F).T @ gy.reshape(-1, C),
            dq.sum(axis=0))
