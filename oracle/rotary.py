"""Norms of rows for each head with the position rotation, in fp64: rows x (B, N, heads, d) to (B, heads, N, d), and the gradients."""
import numpy as np


def _pairs(rot, neighbours):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)


def _rotate(x, angle, rot, neighbours):
    m, n = _pairs(rot, neighbours)
    y = x.copy()
    c, s = np.cos(angle), np.sin(angle)
    y[..., m] = x[..., m] * c - x[..., n] * s
    y[..., n] = x[..., n] * c + x[..., m] * s
    return y


def _scale(x, norm, eps):
    if norm == "none":
        return np.ones(x.shape[:-1] + (1,))
    ss = (x * x).sum(-1, keepdims=True)
    return 1.0 / np.sqrt((ss / x.shape[-1] if norm == "rms" else ss) + eps)


def _angles(positions, inv_freq):
    return np.asarray(positions, dtype=np.float64)[:, :, None, None] * np.asarray(inv_freq, dtype=np.float64)


def forward(x, w, positions, inv_freq, rot, norm, eps, neighbours):
    x = np.asarray(x, dtype=np.float64)
    w = np.ones(x.shape[-1]) if w is None else np.asarray(w, dtype=np.float64)
    y = _rotate(x * _scale(x, norm, eps) * w, _angles(positions, inv_freq), rot, neighbours)
    return y.transpose(0, 2, 1, 3)


def backward(x, w, positions, inv_freq, rot, norm, eps, neighbours, dy):
    """dx (B, N, heads, d) and dw (d)."""
    x = np.asarray(x, dtype=np.float64)
    w = np.ones(x.shape[-1]) if w is None else np.asarray(w, dtype=np.float64)
    r = _scale(x, norm, eps)
    u = _rotate(np.asarray(dy, dtype=np.float64).transpose(0, 2, 1, 3), -_angles(positions, inv_freq), rot, neighbours)
    dw = (u * x * r).sum((0, 1, 2))
    dx = u * w * r
    if norm != "none":
        dx = dx - x * r**3 * (u * w * x).sum(-1, keepdims=True) / (x.shape[-1] if norm == "rms" else 1)
    return dx, dw
