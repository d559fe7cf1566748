"""Oracle: norms of queries and keys per head and their rotation by (t, h, w) positions (test
infrastructure only), float64.

    n   = x / sqrt(mean(x^2) + eps) * weight                  (mean over the channels of one head)
    y   = n with channel pair j of an axis of d_a channels turned by pos_a * theta^(-2 j / d_a)

Pairs are numbered axis by axis (time, height, width); pair j is channels (2j, 2j + 1), or with
``halves`` (j, j + d / 2).  Tokens behind the video (text) and channels behind the axes' are not turned.
The gradients are those of L = sum(dy * y):

    g = turned back dy,   dweight = sum over rows of g * x r,   r = 1 / sqrt(mean(x^2) + eps)
    dx = d/dx sum(g * weight * x r) = r g w - x r^3 mean(g w x)
"""
import numpy as np


def angles(grid, axes, theta=10000.0, origin=(0, 0, 0), head_dim=None):
    """Angle of every pair [N, head_dim / 2] (0 for text tokens and for pairs behind the axes')."""
    f, h, w, text = grid
    out = np.zeros((f * h * w + text, (head_dim or sum(axes)) // 2))
    t, y, x = np.meshgrid(np.arange(f), np.arange(h), np.arange(w), indexing="ij")
    col = 0
    for pos, d_a, o in zip((t, y, x), axes, origin):
        for j in range(d_a // 2):
            out[:f * h * w, col] = (pos.reshape(-1) + float(o)) * float(theta) ** (-2.0 * j / d_a)
            col += 1
    return out


def _pairs(d, halves):
    j = np.arange(d // 2)
    return (j, j + d // 2) if halves else (2 * j, 2 * j + 1)


def rotate(n, ang, halves=False):
    a, b = _pairs(n.shape[-1], halves)
    y = np.empty_like(n)
    y[..., a] = n[..., a] * np.cos(ang) - n[..., b] * np.sin(ang)
    y[..., b] = n[..., a] * np.sin(ang) + n[..., b] * np.cos(ang)
    return y


def norm_rope(x, ang, weight=None, norm=True, eps=1e-6, halves=False):
    """y of rows x [..., N, d]; ang [N, d / 2]."""
    n = np.asarray(x, dtype=np.float64)
    if norm:
        n = n / np.sqrt((n * n).mean(-1, keepdims=True) + eps)
        n = n if weight is None else n * np.asarray(weight, dtype=np.float64)
    return rotate(n, ang, halves)


def norm_rope_grad(dy, x, ang, weight=None, norm=True, eps=1e-6, halves=False):
    """(dx, dweight); dweight None without a norm."""
    g = rotate(np.asarray(dy, dtype=np.float64), -ang, halves)
    if not norm:
        return g, None
    x = np.asarray(x, dtype=np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    gw = g if weight is None else g * np.asarray(weight, dtype=np.float64)
    dx = r * gw - x * r ** 3 * (gw * x).mean(-1, keepdims=True)
    return dx, (g * x * r).reshape(-1, x.shape[-1]).sum(0)
