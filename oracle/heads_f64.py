"""Float64 definitions of the operators around an encoder's attention: the norm of
every head with its rotation by position, and attention over keys of another length.

Plain NumPy, test infrastructure only; nothing here is used by the library.  Rows are
tokens; heads of a row are contiguous.
"""
from __future__ import annotations

import numpy as np


def turn_angles(pos, dim: int, theta: float) -> np.ndarray:
    """[rows, dim / 2] angles pos * theta^(-2 i / dim), in radians."""
    freq = float(theta) ** (-2.0 * np.arange(dim // 2) / dim)
    return np.asarray(pos, np.float64)[:, None] * freq[None, :]


def rotate(x, angles, rotation: str, back: bool = False) -> np.ndarray:
    """x [rows, heads, dim] with pair i turned by angles[row, i].

    rotation: "halves" pairs value i with i + dim / 2, "pairs" 2 i with 2 i + 1,
    "none" leaves x."""
    if rotation == "none":
        return x
    c, s = np.cos(angles)[:, None], np.sin(angles)[:, None]
    s = -s if back else s
    y = np.empty_like(x)
    half = x.shape[-1] // 2
    first = slice(0, half) if rotation == "halves" else slice(0, None, 2)
    second = slice(half, None) if rotation == "halves" else slice(1, None, 2)
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    return y


def head_norm(x, gain, pos, eps, rotation, theta):
    """y = R(pos) (gain * x / sqrt(mean(x^2) + eps)); gain [heads, dim]."""
    rms = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return rotate(gain * x / rms, turn_angles(pos, x.shape[-1], theta), rotation)


def head_norm_backward(x, dy, gain, pos, eps, rotation, theta):
    """(dx, terms): terms summed over rows and the heads of a gain are its gradient."""
    rms = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xhat = x / rms
    dz = rotate(dy, turn_angles(pos, x.shape[-1], theta), rotation, back=True)
    h = dz * gain
    return (h - xhat * (h * xhat).mean(-1, keepdims=True)) / rms, dz * xhat


def cross_attention(q, k, v, lens):
    """(ctx, lse): q [B, Sq, A, D], k, v [B, Skv, Akv, D]; head a reads keys a // (A / Akv).

    lse is log2 of the sum of exp2(log2(e) q.k / sqrt(D)) over the valid keys: -inf, with
    ctx 0, where there are none."""
    B, Sq, A, D = q.shape
    group = A // k.shape[2]
    ctx, lse = np.zeros(q.shape), np.full((B, A, Sq), -np.inf)
    for b in range(B):
        n = int(lens[b])
        for a in range(A if n else 0):
            s = q[b, :, a] @ k[b, :n, a // group].T / np.sqrt(D)
            m = s.max(-1, keepdims=True)
            e = np.exp(s - m)
            total = e.sum(-1, keepdims=True)
            ctx[b, :, a] = e / total @ v[b, :n, a // group]
            lse[b, a] = ((m + np.log(total)) / np.log(2.0))[:, 0]
    return ctx, lse


def cross_attention_backward(q, k, v, dctx, lens):
    """(dq, dk, dv), from the explicit softmax gradient; zeros at keys past lens."""
    B, Sq, A, D = q.shape
    group = A // k.shape[2]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b in range(B):
        n = int(lens[b])
        for a in range(A if n else 0):
            g = a // group
            s = q[b, :, a] @ k[b, :n, g].T / np.sqrt(D)
            e = np.exp(s - s.max(-1, keepdims=True))
            p = e / e.sum(-1, keepdims=True)
            dp = dctx[b, :, a] @ v[b, :n, g].T
            ds = p * (dp - (p * dp).sum(-1, keepdims=True))
            dq[b, :, a] = ds @ k[b, :n, g] / np.sqrt(D)
            dk[b, :n, g] += ds.T @ q[b, :, a] / np.sqrt(D)
            dv[b, :n, g] += p.T @ dctx[b, :, a]
    return dq, dk, dv
