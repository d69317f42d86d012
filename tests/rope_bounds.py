"""How far the norm and rotation of queries and keys may be from the exact ones, element by element.

A result is rounded to bf16 once: u = 2^-8 of it.  Before that all is fp32.  An angle of at most half a turn is rounded to 2^-25 turns (2^-22.3 radians), sine
and cosine of it are off by 2^-22.9 more: under 6 units of 2^-24; a sum of up to 128 squares over 8 or 16 lanes adds at most 20 roundings, halved by
the root, the root itself two; two products with the gain, two and a sum in the rotation: fewer than 2^5 units of 2^-24 of |n_a| + |n_b| in all, F = 2^-18.
Backward the same for the gradient rotated back, once more for the norm's term: 2 F of r (G gain + |x| r^2 mean(G gain |x|)), G the sum of a pair's
|g|.  Gain gradients: F of every term, and a sum of fp32 terms, fewer than 2^8 of them one after the other: 2^-16 of the sum of |terms|."""
import numpy as np

from oracle import skipffn_oracle as O

U, F = 2.0 ** -8, 2.0 ** -18


def pair_sums(x, rot, neighbours):
    """|x_a| + |x_b| in the place of both columns of a rotated pair, |x| elsewhere"""
    y = np.abs(x)
    a, b = O.rope_pairs(rot, neighbours)
    y[..., a] = y[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y


def forward_bound(y, n, rot, neighbours):
    return U * np.abs(y) + F * pair_sums(n, rot, neighbours)


def backward_bounds(x, norm, gain, eps, grad, rot, neighbours, dx):
    """-> bound of grad_x, bound of d_gain"""
    G = pair_sums(grad, rot, neighbours)
    if not norm:
        return U * np.abs(dx) + F * G, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    d_gain = 2.0 ** -16 * (G * np.abs(x) * r).sum((0, 1))
    G = G if gain is None else G * np.abs(gain)
    return U * np.abs(dx) + 2 * F * r * (G + np.abs(x) * r * r * (G * np.abs(x)).mean(-1, keepdims=True)), d_gain
