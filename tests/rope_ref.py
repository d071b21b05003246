"""Norms of heads' rows and rotations by positions, their gradients and how far a kernel may be from them: numpy in 64 bits, angles in 80.

Errors, in units of U = 2^-24 (half a step of 32 bits), each an upper bound:
  angle    the turns of a pair are pos f / 2 pi in 64 bits: f from a power and a division, the product, so 5 half steps of 2^-53 of them; what is
           left of the nearest whole number is rounded to 32 bits (2^-26 turns); the hardware's sine and cosine are 1.3e-7 off at most
  norm     d squares added up in 32 bits, 8 in a row and 4 joins: 12 U of the sum, 6 of its root; with eps, the quotient and the reciprocal root
           (2 U) less than 10 U
  row      weight times cosine, two products, a sum and the factor of the norm: 5 U, of |x_c w_c| + |x_partner w_partner|
  output   half a step of its type
"""
import numpy as np
import torch

U = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}        # half a step of the smallest numbers


def frequencies(d, axis_dims, theta):
    """Axis and frequency of each of the d / 2 pairs."""
    axis = [a for a, dim in enumerate(axis_dims) for _ in range(dim // 2)]
    freq = [theta ** (-2.0 * j / dim) for dim in axis_dims for j in range(dim // 2)]
    rest = d // 2 - len(axis)
    return np.array(axis + [0] * rest, dtype=int), np.array(freq + [0.0] * rest, dtype=np.longdouble)


def partners(d, halves):
    """The channel each channel is paired with, its pair, and the sign of the partner's share."""
    c = np.arange(d)
    if halves:
        return (c + d // 2) % d, c % (d // 2), np.where(c < d // 2, -1.0, 1.0)
    return c ^ 1, c // 2, np.where(c % 2 == 0, -1.0, 1.0)


class Rotation:
    """The rotation of tokens at `pos` [..., tokens, axes]; rows are [..., tokens, heads, d]."""

    def __init__(self, pos, d, axis_dims, theta=10000.0, halves=False, freq=None):
        axis, f = frequencies(d, axis_dims, theta)
        if freq is not None:
            f = np.concatenate([np.asarray(freq, dtype=np.longdouble), np.zeros(d // 2 - len(freq), dtype=np.longdouble)])
        self.d = d
        self.partner, pair, self.sign = partners(d, halves)
        if len(axis_dims) == 0:
            angle = np.zeros(pos.shape[:-1] + (d // 2,), dtype=np.longdouble)
        else:
            angle = pos.astype(np.longdouble)[..., axis] * f
        angle = angle[..., None, :][..., pair]
        self.cos, self.sin = np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64)
        self.error = 1.3e-7 + 2 * np.pi * 2.0 ** -26 + 5 * 2.0 ** -53 * np.abs(angle).astype(np.float64)

    def turn(self, y):
        return y * self.cos + y[..., self.partner] * self.sign * self.sin

    def back(self, z):
        return z * self.cos - z[..., self.partner] * self.sign * self.sin

    def size(self, y):
        """What errors of a rotation are relative to."""
        return np.abs(y) + np.abs(y)[..., self.partner]


def scale(x, eps):
    return 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def forward(rot, x, w=None, eps=1e-6):
    """(rows, how far 32 bits may be from them)."""
    y = x if w is None else x * scale(x, eps) * w
    return rot.turn(y), rot.size(y) * (rot.error + (15 if w is not None else 3) * U)


def rounded(value, error, dtype):
    """How far the rounded output may be."""
    return error + HALF_STEP[dtype] * (np.abs(value) + error) + LEAST[dtype]


def backward(rot, x, dz, w=None, eps=1e-6):
    """(dx, its error, dw, its error); heads and tokens are all axes of x but the last."""
    g = rot.back(dz)
    g_error = rot.size(dz) * (rot.error + 3 * U)
    if w is None:
        return g, g_error, None, None
    r = scale(x, eps)
    n = x * r
    size = rot.size(dz) * np.abs(w)
    mean = (g * w * n).mean(-1, keepdims=True)
    dx = r * (g * w - n * mean)
    # of dx: the factor and n (10 U each, n twice in the second term), the mean (13 U more), products and the sum (4 U)
    most = r * (size + np.abs(n) * (size * np.abs(n)).mean(-1, keepdims=True))
    dx_error = most * (rot.error.max(-1, keepdims=True) + 45 * U)
    rows = tuple(range(x.ndim - 1))
    dw = (g * n).sum(rows)
    # of dw: g and n (14 U), and sums of 32 bits over the heads of a token at most, then 64 and two roundings
    dw_error = ((rot.size(dz) * np.abs(n)) * (rot.error + (14 + 3 + x.shape[-2]) * U)).sum(rows)
    return dx, dx_error, dw, dw_error
