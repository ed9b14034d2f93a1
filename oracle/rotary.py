"""Head norms and rotary positions in 64 bits, from their definition: the checker of the padoc_*_rotary calls.
Shares no code with the library."""
import numpy as np


def _pairs(rot, adjacent):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)


def angles(pos, inv_freq, axis_of):
    """[rows][pairs] fp64: position on the pair's axis x frequency."""
    pos = np.asarray(pos, np.float64)
    return pos[:, np.asarray(axis_of, np.int64)] * np.asarray(inv_freq, np.float64)[None]


def forward(x, weight, eps, angle, adjacent=False, amplitude=1.0):
    """x [rows][heads][d] -> (z, scale of each value's error: |u| + |v| over its pair, times |amplitude|)."""
    y = np.asarray(x, np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    i, j = _pairs(2 * angle.shape[1], adjacent)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    z, size = y.copy(), np.abs(y)
    z[..., i] = amplitude * (y[..., i] * c - y[..., j] * s)
    z[..., j] = amplitude * (y[..., j] * c + y[..., i] * s)
    both = abs(amplitude) * (np.abs(y[..., i]) + np.abs(y[..., j]))
    size[..., i] = both
    size[..., j] = both
    return z, size


def turn_back(dz, angle, adjacent=False, amplitude=1.0):
    """The upstream gradient turned by the opposite angles, and the scale of its error."""
    return forward(dz, None, 0.0, -angle, adjacent, amplitude)


def backward(dz, x, weight, eps, angle, adjacent=False, amplitude=1.0):
    """Returns (dx, scale of dx's error, dweight, sum of the magnitudes of dweight's terms); without a weight
    the last two are None."""
    g, size = turn_back(dz, angle, adjacent, amplitude)
    if weight is None:
        return g, size, None, None
    x, w = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    h = x * r
    dx = r * (w * g - h * (w * g * h).mean(-1, keepdims=True))
    scale = r * (np.abs(w) * size + np.abs(h) * (np.abs(w * h) * size).mean(-1, keepdims=True))
    return dx, scale, (g * h).sum((0, 1)), (size * np.abs(h)).sum((0, 1))
