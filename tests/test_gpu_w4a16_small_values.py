"""W4A16 layers behind a norm that gives small values: by gamma, by an eps that is more than the row, or in some rows only.  What goes in as two halves keeps its 22
bits, or 2^-38 of the row's largest value where that is more."""
import numpy as np
import pytest
import torch

import _fp16_layer_ref as ref
import paper_2310_19102_amd as atom
from test_gpu_w4a16 import case, close, gpu

pytestmark = pytest.mark.gpu

EPS = 1e-5


def activations(x, gamma, eps, idx):
    """(xr in 64 bits, bound on what the library's xr is off by): as ref.activations, but for what two halves of a row that is brought to 2^14 by a power of two
    lose: half a step of lo, 2^-25 of 2^14 or (where the row's largest value comes out a rounding smaller) a little more."""
    x = x.astype(np.float64)
    x = x / np.sqrt((x * x).mean(1, keepdims=True) + eps) * gamma.astype(np.float64)
    off = (2.0 ** -22 + (x.shape[1] / 512 + 17) * 2.0 ** -24) * np.abs(x) + 2.0 ** -38 * np.abs(x).max(1, keepdims=True)
    return (x, off) if idx is None else (x[:, idx], off[:, idx])


def inputs(M, N, K, kind, matrices):
    """Weights so large that results are normal numbers."""
    x, gamma, idx, w, rng = case(M, N, K, 128, matrices, seed=7)
    x = rng.standard_normal((M, K)).astype(np.float16)
    size = 1.0
    if kind == "gamma":
        gamma, size = (gamma.astype(np.float64) * 2e-5).astype(np.float16), 2e-5
    elif kind == "eps":                                       # values of some 2^-22 behind an eps of 2^-16
        x, size = (x.astype(np.float64) * 2.0 ** -22).astype(np.float16), 2.0 ** -22 / EPS ** 0.5
    elif kind == "rows":
        x[::2] = (x[::2].astype(np.float64) * 2.0 ** -22).astype(np.float16)
        size = 2.0 ** -22 / EPS ** 0.5
    else:                                                     # one large channel among small ones
        gamma = (gamma.astype(np.float64) * 1e-4).astype(np.float16)
        gamma[K // 3] = 1
        size = 1e-4
    scale = np.float16(min(60000, 0.02 / size / K ** 0.5 * (1 if kind != "rows" else 0.02)))
    w = [(q4, np.clip(q8, -20, 20), (scale * (0.5 + rng.random(s.shape))).astype(np.float16)) for q4, q8, s in w]
    return x, gamma, idx, w


SIZES = [(1, 100, 1024), (1, 50, 24576), (3, 77, 4096), (8, 300, 8192), (8, 9001, 4096), (9, 65, 640), (16, 130, 8192), (20, 300, 1024), (40, 200, 4224), (64, 520, 2048)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("kind", ["gamma", "eps", "rows", "channel"])
@pytest.mark.parametrize("index", [False, True])
def test_linear(M, N, K, kind, index):
    x, gamma, idx, (w,) = inputs(M, N, K, kind, 1)
    idx = idx if index else None
    y, tol = ref.sums(*activations(x, gamma, EPS, idx), w)
    tol = ref._rounded(y, tol)
    assert np.abs(y).max() < 60000 and np.median(np.abs(y)) > 2.0 ** -10
    close(atom.atom_w4a16_linear(gpu(x), gpu(gamma), EPS, gpu(idx), *gpu(w)), y, tol)


@pytest.mark.parametrize("M,N,K", [(1, 100, 1024), (3, 77, 4096), (8, 9001, 4096), (9, 65, 640), (16, 130, 8192), (20, 300, 1024), (40, 200, 4224)])
@pytest.mark.parametrize("kind", ["gamma", "rows"])
def test_swiglu(M, N, K, kind):
    x, gamma, idx, (gate, up) = inputs(M, N, K, kind, 2)
    xr, off = activations(x, gamma, EPS, idx)
    (g, dg), (u, du) = ref.sums(xr, off, gate), ref.sums(xr, off, up)
    act = g / (1 + np.exp(-g))
    h = act * u
    # as in ref.swiglu: silu' lies between -0.1 and 1.1; exp, quotient and products in fp32
    tol = ref._rounded(h, 1.1 * dg * (np.abs(u) + du) + np.abs(act) * du + 16 * 2.0 ** -24 * np.abs(h))
    assert np.abs(h).max() < 60000
    close(atom.atom_w4a16_swiglu(gpu(x), gpu(gamma), EPS, gpu(idx), gpu(gate), gpu(up)), h, tol)


@pytest.mark.parametrize("M", [1, 6, 12, 30])
def test_rows_of_zeros_and_of_what_is_not_finite_between_them(M):
    """A row's power of two is its own: zeros give zeros, also with eps = 0 NaN only there."""
    N, K = 90, 768
    x, gamma, idx, (w,) = inputs(M, N, K, "gamma", 1)
    if M > 2:
        x[0], x[1, 9] = 0, np.nan
    rows = list(range(2, M)) if M > 2 else [0]
    y, tol = ref.sums(*activations(x[rows], gamma, EPS, idx), w)
    got = atom.atom_w4a16_linear(gpu(x), gpu(gamma), EPS, gpu(idx), *gpu(w))
    close(got[rows], y, ref._rounded(y, tol))
    if M > 2:
        assert bool((got[0] == 0).all()) and bool(torch.isnan(got[1]).all())
        got = atom.atom_w4a16_linear(gpu(x), gpu(gamma), 0.0, gpu(idx), *gpu(w))
        y, tol = ref.sums(*activations(x[rows], gamma, 0.0, idx), w)
        close(got[rows], y, ref._rounded(y, tol))
        assert bool(torch.isnan(got[:2]).all())
