"""64-bit references (numpy, CPU) of the operators around a mixer with one decay a head: the recurrence step by step with its reverse-mode
derivative, rotary positions, and layer norm with the output gate.  They share no code with the library.

Sequences are [B, H, T, d] here; scan orders, memory orders and lengths are taken apart by ``visits``.
"""
import numpy as np


def visits(T, grid_h, grid_w, scan_dir, length=None):
    """Token numbers in the order of the scan (row forward, row reversed, column forward, column reversed)."""
    n = np.arange(T if length is None else length)
    if scan_dir >= 2:
        n = np.arange(T).reshape(grid_h, grid_w).T.reshape(-1)
    return n[::-1] if scan_dir & 1 else n


def decay_fwd(q, k, v, g, s0):
    """q, k [N,T,dk], v [N,T,dv], g [N,T], s0 [N,dk,dv], all in visiting order: outputs [N,T,dv] and all states [N,T+1,dk,dv]."""
    N, T, dk = q.shape
    S = np.zeros((N, T + 1, dk, v.shape[2]))
    S[:, 0] = s0
    o = np.zeros((N, T, v.shape[2]))
    for t in range(T):
        S[:, t + 1] = np.exp(g[:, t])[:, None, None] * S[:, t] + k[:, t, :, None] * v[:, t, None, :]
        o[:, t] = np.matmul(q[:, t, None], S[:, t + 1])[:, 0]
    return o, S


def decay_bwd(q, k, v, g, S, do, ds_last):
    """Gradients dq, dk, dv, dg and ds0 by the chain rule through decay_fwd's steps, from the last to the first."""
    N, T, dk = q.shape
    dq, dk_, dv, dg = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(g.shape)
    G = ds_last.copy()                                    # dL/dS after step t, from the steps behind it
    for t in range(T - 1, -1, -1):
        dq[:, t] = np.matmul(S[:, t + 1], do[:, t, :, None])[..., 0]
        G = G + q[:, t, :, None] * do[:, t, None, :]
        dk_[:, t] = np.matmul(G, v[:, t, :, None])[..., 0]
        dv[:, t] = np.matmul(k[:, t, None], G)[:, 0]
        G = np.exp(g[:, t])[:, None, None] * G
        dg[:, t] = (G * S[:, t]).sum((1, 2))
    return dq, dk_, dv, dg, G


def rope(x, positions, sections, base, adjacent, inverse):
    """x [B,H,T,d], positions [B,T,axes]."""
    y = x.astype(np.float64).copy()
    at = 0
    for a, w in enumerate(sections):
        for i in range(w // 2):
            c0, c1 = (at + 2 * i, at + 2 * i + 1) if adjacent else (at + i, at + i + w // 2)
            ang = positions[:, None, :, a].astype(np.float64) * float(base) ** (-2.0 * i / w) * (-1.0 if inverse else 1.0)
            u, v = x[..., c0].astype(np.float64), x[..., c1].astype(np.float64)
            y[..., c0], y[..., c1] = u * np.cos(ang) - v * np.sin(ang), v * np.cos(ang) + u * np.sin(ang)
        at += w
    return y


def _sigmoid(r):
    return 1.0 / (1.0 + np.exp(-r))


def norm_fwd(x, w, b, eps, r=None):
    """x [..., H, D] with the head before the channels, w, b [H, D]: outputs, normalised rows and 1 / sqrt(var + eps)."""
    mean = x.mean(-1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    n = (x - mean) * rstd
    y = n * w + b
    return (y if r is None else y * r * _sigmoid(r)), n, rstd


def norm_bwd(x, w, b, eps, do, r=None):
    """dx, dr (or None), dw, db; the sums of the last two over all axes but [H, D]."""
    _, n, rstd = norm_fwd(x, w, b, eps)
    D = x.shape[-1]
    dr = None
    dy = do
    if r is not None:
        sg = _sigmoid(r)
        dr = do * (n * w + b) * (sg + r * sg * (1 - sg))
        dy = do * r * sg
    dn = dy * w
    # dn through the row's mean and variance: n = (x - mean) rstd
    dvar = (dn * (x - x.mean(-1, keepdims=True))).sum(-1, keepdims=True) * -0.5 * rstd ** 3
    dxc = dn * rstd + 2.0 / D * (x - x.mean(-1, keepdims=True)) * dvar
    dx = dxc - dxc.mean(-1, keepdims=True)
    over = tuple(range(x.ndim - 2))
    return dx, dr, (dy * n).sum(over), dy.sum(over)
