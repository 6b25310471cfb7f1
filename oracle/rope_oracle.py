"""Plain definition of rotary positions and of the norm of every head with the
rotation, forward and backward (numpy, fp64 with angles in extended precision,
CPU): test infrastructure only, shares no code with the GPU path."""
import numpy as np


def angles(pos, freq):
    """cos and sin [N, L, 1, rot / 2] of position times frequency (radians)."""
    p = np.asarray(pos, np.int64).astype(np.longdouble)[:, :, None, None] * np.asarray(freq, np.longdouble)
    return np.cos(p).astype(np.float64), np.sin(p).astype(np.float64)


def _pairs(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(x, pos, freq, interleaved, amplitude=1.0, transpose=False):
    c, s = angles(pos, freq)
    s = -s if transpose else s
    a, b = _pairs(2 * len(freq), interleaved)
    y = np.array(x, np.float64)
    y[..., a] = amplitude * (x[..., a] * c - x[..., b] * s)
    y[..., b] = amplitude * (x[..., a] * s + x[..., b] * c)
    return y


def rstd(x, eps):
    return 1.0 / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)


def forward(x, pos, freq, interleaved=False, amplitude=1.0, norm=False, w=None, eps=1e-6):
    u = np.asarray(x, np.float64)
    if norm:
        u = u * rstd(u, eps) * (1.0 if w is None else np.asarray(w, np.float64))
    return rotate(u, pos, freq, interleaved, amplitude)


def backward(dy, x, pos, freq, interleaved=False, amplitude=1.0, norm=False, w=None, eps=1e-6):
    """(dx, dw); dw None without a weight."""
    g = rotate(np.asarray(dy, np.float64), pos, freq, interleaved, amplitude, True)
    if not norm:
        return g, None
    x = np.asarray(x, np.float64)
    r = rstd(x, eps)
    hat = x * r
    t = g if w is None else g * np.asarray(w, np.float64)
    dx = r * (t - hat * np.mean(t * hat, -1, keepdims=True))
    return dx, None if w is None else np.sum(g * hat, (0, 1, 2))
