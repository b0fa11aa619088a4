"""64-bit references (numpy, CPU) of what stands around the mixer in a block: the gated recurrence of channels step by step with its reverse-mode
derivative, the root-mean-square norm of queries and keys, and the gated feed-forward product.  They share no code with the library.
"""
import math

import numpy as np


def log_gate(z, tau=None):
    """Logarithms of the gates: z itself, or those of sigmoid(z)^(1/tau); and their derivative by z."""
    z = np.asarray(z, np.float64)
    if tau is None:
        return z, np.ones_like(z)
    e = np.exp(-np.abs(z))
    return (np.minimum(z, 0.0) - np.log1p(e)) / tau, np.where(z > 0, e, 1.0) / (1.0 + e) / tau


def recur_fwd(x, lg, rest, h0):
    """x, lg [B,T,D] in visiting order, h0 [B,D]: the states [B,T+1,D], the first one h0."""
    h = np.zeros((x.shape[0], x.shape[1] + 1, x.shape[2]))
    h[:, 0] = h0
    for t in range(x.shape[1]):
        h[:, t + 1] = np.exp(lg[:, t]) * h[:, t] + (x[:, t] * -np.expm1(lg[:, t]) if rest else x[:, t])
    return h


def recur_bwd(x, lg, rest, h, do, dh_last):
    """Gradients dx, dlg and dh0 by the chain rule through recur_fwd's steps, from the last to the first."""
    dx, dlg = np.zeros(x.shape), np.zeros(x.shape)
    G = np.array(dh_last, np.float64)
    for t in range(x.shape[1] - 1, -1, -1):
        G = G + do[:, t]
        a = np.exp(lg[:, t])
        dx[:, t] = G * -np.expm1(lg[:, t]) if rest else G
        dlg[:, t] = G * a * h[:, t] - (G * a * x[:, t] if rest else 0.0)
        G = G * a
    return dx, dlg, G


def rms_fwd(x, w, eps):
    """x [..., d], w [d]: the rows over their root mean square, times w; and 1 / root."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r * w, r


def rms_bwd(x, w, eps, dy):
    """dx and dw (summed over all rows)."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dn = dy * w
    # through the root: r' = -r^3 / d * x
    dx = dn * r - x * r ** 3 * (dn * x).mean(-1, keepdims=True)
    return dx, (dy * x * r).reshape(-1, x.shape[-1]).sum(0)


def activation(kind, g):
    """silu, gelu (by the normal distribution) or gelu_tanh, and its derivative."""
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if kind == "gelu":
        phi = np.vectorize(lambda t: 0.5 * math.erfc(-t / math.sqrt(2.0)), otypes=[np.float64])(g) if g.size else g * 0.0
        return g * phi, phi + g * np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    c = math.sqrt(2.0 / math.pi)
    t = np.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * g * g)


def glu_fwd(x, wg, wu, kind):
    """x [M,K], wg, wu [F,K]: act(x wg^T) * (x wu^T)."""
    return activation(kind, x @ wg.T)[0] * (x @ wu.T)


def glu_bwd(x, wg, wu, kind, do):
    g, u = x @ wg.T, x @ wu.T
    act, slope = activation(kind, g)
    dg, du = do * u * slope, do * act
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x
