"""Norms and rotation of heads in 64 bits (include/tahq_heads.h), forward and backward, on the CPU: NumPy only."""
import math

import numpy as np


def frequencies(rotated, base=10000.0, scaling="plain", factor=1.0, original=4096, low=1.0, high=32.0):
    """Radians per position of every pair."""
    if scaling == "stretched" and rotated > 2:
        base = base * factor ** (rotated / (rotated - 2))
    f = np.array([base ** (-2.0 * i / rotated) for i in range(rotated // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        k = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0, 1)
        f = k * f + (1 - k) * f / factor
    return f


def _places(rotated, pairs):
    """Channels of the first and of the second numbers of the pairs."""
    return (np.arange(0, rotated, 2), np.arange(1, rotated, 2)) if pairs else (np.arange(rotated // 2), rotated // 2 + np.arange(rotated // 2))


def turn(x, positions, f, rotated, pairs, magnitude, back=False):
    """[tokens, heads, head] with its pairs turned; and the sum of the terms' magnitudes."""
    a, b = _places(rotated, pairs)
    # modulo a turn in integers would be exact; in 64 bits positions below 2^24 are off by 2^-28 at most, as numbers of 2^25 radians
    t = positions.astype(np.float64)[:, None, None] * f
    c, s = magnitude * np.cos(t), magnitude * np.sin(t) * (-1 if back else 1)
    y, size = x.astype(np.float64).copy(), np.abs(x.astype(np.float64))
    xa, xb = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = xa * c - xb * s, xa * s + xb * c
    size[..., a] = size[..., b] = abs(magnitude) * (np.abs(xa) + np.abs(xb))
    return y, size


def forward(x, w, positions, f, rotated, pairs, eps, magnitude):
    n = x.astype(np.float64)
    if w is not None:
        n = n / np.sqrt(np.square(n).mean(-1, keepdims=True) + eps) * w
    return turn(n, positions, f, rotated, pairs, magnitude)


def backward(grad, x, w, positions, f, rotated, pairs, eps, magnitude):
    """(gradient of x, its size, gradient of w, its size); sizes are sums of the terms' magnitudes."""
    g, size = turn(grad, positions, f, rotated, pairs, magnitude, back=True)
    if w is None:
        return g, size, None, None
    x = x.astype(np.float64)
    rstd = 1 / np.sqrt(np.square(x).mean(-1, keepdims=True) + eps)
    n = x * rstd
    dw, dw_size = (g * n).sum((0, 1)), (size * np.abs(n)).sum((0, 1))
    u, u_size = g * w, size * np.abs(w)
    return (rstd * (u - n * (u * n).mean(-1, keepdims=True)), rstd * (u_size + np.abs(n) * (u_size * np.abs(n)).mean(-1, keepdims=True)), dw, dw_size)
