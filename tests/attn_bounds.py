"""How far a bf16 kernel's attention may be from the exact one, element by element.

A rounding to bf16 is off by at most u = 2^-8 of the value.  Rounded are: the weights P before they meet v (and
before they meet grad_out), dS before it meets k and q, and every result once.  All else is fp32: f covers the weights'
relative error from scores (128 products of at most a few units, 2^-24 each, times |q| . |k| scale log2(e) of about 12:
1e-4 = 2^-13) and from the exponential; p the products of grad_out and v (128 terms of 2^-24: 2^-17).  With A = sum_j P |v|:
    out     (u + f) A + u |out|
    delta   |grad_out| . (error of out), as it is taken from the rounded out
    dS      P (error of delta + p |grad_out| . |v|) + (u + f) |dS|
    dq      scale sum_j (error of dS) |k| + u |dq|;   dk the same over queries
    dv      (u + f) sum_i P |grad_out| + u |dv|
and 2^-6 of that again for products of two of these."""
import numpy as np

U, F, P16 = 2.0 ** -8, 2.0 ** -12, 2.0 ** -16
SLACK = 1 + 2.0 ** -6


def out_bound(P, v, out):
    """P [H, nq, nk], v [nk, Hkv, D], out [nq, H, D]"""
    rep = P.shape[0] // v.shape[1]
    A = np.stack([P[h] @ np.abs(v[:, h // rep]) for h in range(P.shape[0])], axis=1) if len(v) else np.zeros(out.shape)
    return SLACK * ((U + F) * A + U * np.abs(out))


def grad_bounds(q, k, v, g, scale, b):
    """b: what the oracle's attn_backward_real gave -> bounds of dq, dk, dv"""
    H, Hkv = q.shape[1], k.shape[1]
    e_out = out_bound(b["P"], v, b["out"])
    eq, ek, ev = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for h in range(H):
        kh = h // (H // Hkv)
        e_delta = (np.abs(g[:, h]) * (e_out[:, h] + P16 * np.abs(b["out"][:, h]))).sum(axis=1, keepdims=True)
        E = b["P"][h] * (e_delta + P16 * (np.abs(g[:, h]) @ np.abs(v[:, kh]).T)) + (U + F) * np.abs(b["dS"][h])
        eq[:, h] = scale * (E @ np.abs(k[:, kh]))
        ek[:, kh] += scale * (E.T @ np.abs(q[:, h]))
        ev[:, kh] += (U + F) * (b["P"][h].T @ np.abs(g[:, h]))
    return {n: SLACK * (e + U * np.abs(b[n])) for n, e in (("dq", eq), ("dk", ek), ("dv", ev))}


def assert_within(got, want, bound, what):
    off = np.abs(got - want)
    bad = ~(off <= bound + 1e-30)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} elements, first at {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]} for {want[bad][0]}, off {off[bad][0]:.3g}, allowed {bound[bad][0]:.3g}")
