"""The operators of a decoding layer in fp16 activations, in plain numpy: the turn in IEEE fp32 steps (bit-exact) and in 64
bits, linear layers on 4-bit weights in 64 bits with the error that the library's arithmetic may have."""
import numpy as np


def table(n_pos, n_pairs, base=10000.0):
    angle = np.arange(n_pos)[:, None] * base ** (-np.arange(n_pairs) / n_pairs)[None, :]
    return np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)


def turned(x, positions, tab, axis=None, interleaved=False, transposed=False, dtype=np.float32):
    """x [T, heads, D] turned, in `dtype`: every product and sum is rounded once."""
    P, n, _ = tab.shape
    pos = np.atleast_2d(positions)[list(axis) if axis is not None else [0] * n]          # [pairs, T]
    ok = (pos >= 0) & (pos < P)
    c, s = (np.where(ok, tab[np.where(ok, pos, 0), np.arange(n)[:, None], i], np.nan if i == 0 else 0).T[:, None].astype(dtype) for i in (0, 1))
    s = np.where(np.isnan(c), np.nan, -s if transposed else s).astype(dtype)
    y = x.astype(dtype)
    lo, hi = (np.s_[..., 0:2 * n:2], np.s_[..., 1:2 * n:2]) if interleaved else (np.s_[..., :n], np.s_[..., n:2 * n])
    a, b = y[lo].copy(), y[hi].copy()
    with np.errstate(invalid="ignore"):
        y[lo], y[hi] = a * c - b * s, b * c + a * s
    return y


def codes_of(q4, q8):
    """[N, K] whole numbers."""
    low, high = (q4 & 15).astype(np.int32), (q4 >> 4).astype(np.int32)
    both = np.stack([low, high], -1).reshape(q4.shape[0], -1)
    return np.concatenate([both - 16 * (both > 7), q8.astype(np.int32)], 1)


def activations(x, gamma, eps, idx):
    """(xr in 64 bits, bound on what the library's xr is off by)."""
    x = x.astype(np.float64)
    off = np.zeros_like(x)
    if gamma is not None:
        x = x / np.sqrt((x * x).mean(1, keepdims=True) + eps) * gamma.astype(np.float64)
        # two halves (2^-22 of itself, 2^-25 below the normal numbers); before that the sum of squares in fp32, at most K / 256 + 24 additions
        # behind one another (half of their error in the root), and five more roundings
        off = (2.0 ** -22 + (x.shape[1] / 512 + 17) * 2.0 ** -24) * np.abs(x) + 2.0 ** -25
    return (x, off) if idx is None else (x[:, idx], off[:, idx])


def sums(xr, off, weights):
    """(the sum over all groups in 64 bits, bound on the library's fp32 sum's error)."""
    q4, q8, scale = weights
    w = codes_of(q4, q8).astype(np.float64) * np.repeat(scale.astype(np.float64), 128, 1)
    y, mass = xr @ w.T, np.abs(xr) @ np.abs(w).T
    # products are exact; the additions inside the matrix instruction and after it may each lose one step of the sum so far
    return y, off @ np.abs(w).T + (128 + scale.shape[1] + 16) * 2.0 ** -23 * (mass + off @ np.abs(w).T)


def _rounded(y, tol):
    return tol + 2.0 ** -11 * (np.abs(y) + tol) + 2.0 ** -25


def linear(x, gamma, eps, idx, weights, residual=None):
    """(y [M, N] in 64 bits, tolerance)."""
    y, tol = sums(*activations(x, gamma, eps, idx), weights)
    if residual is not None:
        y = y + residual.astype(np.float64)
        tol = tol + 2.0 ** -24 * (np.abs(y) + tol)
    return y, _rounded(y, tol)


def swiglu(x, gamma, eps, idx, gate, up):
    xr, off = activations(x, gamma, eps, idx)
    (g, dg), (u, du) = sums(xr, off, gate), sums(xr, off, up)
    act = g / (1 + np.exp(-g))
    h = act * u
    # silu' lies between -0.1 and 1.1; exp, quotient and products in fp32
    tol = 1.1 * dg * (np.abs(u) + du) + np.abs(act) * du + 16 * 2.0 ** -24 * np.abs(h)
    return h, _rounded(h, tol)
