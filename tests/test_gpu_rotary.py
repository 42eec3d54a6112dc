"""Rotary positions against IEEE fp32 steps in numpy, bit for bit, and against the formula in 64 bits."""
import numpy as np
import pytest
import torch

import _fp16_layer_ref as ref
import paper_2310_19102_amd as atom

pytestmark = pytest.mark.gpu


def case(T, heads, D, R, axes, interleaved, P=97, seed=0):
    rng = np.random.default_rng([T, heads, D, R, axes, interleaved, seed])
    x = rng.standard_normal((T, heads, D)).astype(np.float16)
    pos = rng.integers(0, P, (axes, T)).astype(np.int32)
    axis = None if axes == 1 else rng.integers(0, axes, R // 2).tolist()
    return x, pos if axes > 1 else pos[0], ref.table(P, R // 2), axis


def gpu(*arrays):
    return [torch.from_numpy(a).cuda() if isinstance(a, np.ndarray) else a for a in arrays]


def same(got, want):
    got, want = got.cpu().numpy(), want.astype(np.float16)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    there = ~np.isnan(want)
    assert np.array_equal(got[there].view(np.uint16), want[there].view(np.uint16))


@pytest.mark.parametrize("T,heads,D,R,axes", [
    (1, 1, 8, 8, 1), (1, 64, 128, 128, 1), (3, 5, 64, 64, 3), (2, 7, 80, 32, 2), (63, 72, 128, 128, 3), (300, 20, 64, 16, 4), (17, 3, 256, 256, 4),
    (129, 1, 128, 64, 1), (40, 9, 96, 96, 1), (4099, 2, 64, 32, 2), (257, 33, 24, 8, 1)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("transposed", [False, True])
def test_bits(T, heads, D, R, axes, interleaved, transposed):
    x, pos, tab, axis = case(T, heads, D, R, axes, interleaved)
    want = ref.turned(x, pos, tab, axis, interleaved, transposed)
    xd, pd, td = gpu(x, pos, tab)
    same(atom.atom_rotary(xd, pd, td, axis, interleaved, transposed), want)
    # in place, and between slices of larger tensors: nothing else is touched
    wide, out = torch.full((T, heads + 3, D), 7.0, dtype=torch.float16, device="cuda"), torch.full((T, heads + 2, D), 9.0, dtype=torch.float16, device="cuda")
    wide[:, 1:1 + heads] = xd
    atom.atom_rotary(wide[:, 1:1 + heads], pd, td, axis, interleaved, transposed, out=out[:, 2:])
    same(out[:, 2:], want)
    assert bool((out[:, :2] == 9).all()) and torch.equal(wide[:, 1:1 + heads], xd)
    atom.atom_rotary(wide[:, 1:1 + heads], pd, td, axis, interleaved, transposed, out=wide[:, 1:1 + heads])
    same(wide[:, 1:1 + heads], want)
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, 1 + heads:] == 7).all())
    # the formula: the table's entries, two products and a sum are rounded to fp32, the result to fp16
    exact = ref.turned(x, pos, tab, axis, interleaved, transposed, np.float64)
    assert (np.abs(want.astype(np.float16) - exact) <= 2.0 ** -11 * np.abs(exact) + 2.0 ** -25 + 4 * 2.0 ** -24 * np.abs(x).max() * 2).all()


@pytest.mark.parametrize("n_pos,n_pairs", [(1, 1), (5, 4), (1000, 64), (70001, 128), (0, 8)])
def test_table(n_pos, n_pairs):
    freq = 10000.0 ** (-np.arange(n_pairs) / n_pairs)
    got = atom.atom_rotary_table(torch.from_numpy(freq).cuda(), n_pos).cpu().numpy().astype(np.float64)
    angle = np.arange(n_pos)[:, None] * freq[None]
    # one rounding to fp32 of values that two libraries give to a few ulps of 64 bits
    assert got.shape == (n_pos, n_pairs, 2)
    for i, f in enumerate((np.cos, np.sin)):
        assert (np.abs(got[..., i] - f(angle)) <= 2.0 ** -24 * np.abs(f(angle)) + 2.0 ** -50 * 8).all()


@pytest.mark.parametrize("axes", [1, 2])
def test_positions_outside_the_table_give_nan_in_what_they_turn(axes):
    T, heads, D, R, P = 12, 5, 64, 32, 10
    x, pos, tab, axis = case(T, heads, D, R, axes, False, P)
    rows = pos if axes > 1 else pos[None]
    rows[0, 2], rows[0, 7], rows[-1, 9], rows[-1, 11] = -1, P, 2 ** 31 - 1, -2 ** 31
    want = ref.turned(x, pos, tab, axis)
    assert np.isnan(want).any() and not np.isnan(want[0]).any()
    same(atom.atom_rotary(*gpu(x, pos, tab), axis), want)


def test_values_that_are_not_finite_stay_with_their_pairs():
    x, pos, tab, _ = case(6, 3, 64, 64, 1, False)
    x[1, 0, 5], x[2, 1, 40], x[3, 2, 63] = np.inf, np.nan, -np.inf
    pos[3] = 0
    with np.errstate(invalid="ignore"):
        want = ref.turned(x, pos, tab)
    assert np.isfinite(want).sum() >= want.size - 6
    same(atom.atom_rotary(*gpu(x, pos, tab)), want)


def test_no_tokens_and_one_position():
    x, pos, tab, _ = case(0, 4, 64, 64, 1, False)
    assert atom.atom_rotary(*gpu(x, pos, tab)).shape == (0, 4, 64)
    x, pos, tab, _ = case(9, 4, 64, 64, 1, False, P=1)
    same(atom.atom_rotary(*gpu(x, pos, tab)), x)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(interleaved):
    """f(x) = sum(g * turned(x)) is linear: its differences are its gradient up to the roundings of fp16, which sums of
    whole numbers of quarter turns do not have."""
    T, heads, D, R = 4, 2, 16, 8
    rng = np.random.default_rng(5)
    tab = np.stack([np.array([1.0, 0, -1, 0]), np.array([0, 1.0, 0, -1])], -1).astype(np.float32)[:, None].repeat(R // 2, 1)
    pos = rng.integers(0, 4, T).astype(np.int32)
    x, g = (rng.integers(-4, 5, (T, heads, D)).astype(np.float16) for _ in range(2))
    xd, pd, td, gd = gpu(x, pos, tab, g)
    grad = atom.atom_rotary(gd, pd, td, interleaved=interleaved, transposed=True).cpu().numpy().astype(np.float64)
    for _ in range(40):
        t, h, c = rng.integers(T), rng.integers(heads), rng.integers(D)
        f = []
        for step in (1.0, -1.0):
            y = xd.clone()
            y[t, h, c] += step
            f.append(float((gd.double() * atom.atom_rotary(y, pd, td, interleaved=interleaved).double()).sum()))
        assert (f[0] - f[1]) / 2 == grad[t, h, c]
    # general angles: the two ways are each other's transpose
    x, pos, tab, _ = case(50, 6, 64, 64, 1, interleaved)
    g = np.random.default_rng(6).standard_normal(x.shape).astype(np.float16)
    a = (ref.turned(x, pos, tab, None, interleaved, False, np.float64) * g).sum()
    back = atom.atom_rotary(*gpu(g, pos, tab), interleaved=interleaved, transposed=True).cpu().numpy().astype(np.float64)
    assert abs(a - (back * x).sum()) <= (2.0 ** -11 * np.abs(back * x) + 2.0 ** -25 * np.abs(x) + 2.0 ** -21 * np.abs(x)).sum()
    # there and back
    y = atom.atom_rotary(atom.atom_rotary(*gpu(x, pos, tab), interleaved=interleaved), *gpu(pos, tab), interleaved=interleaved, transposed=True)
    assert (np.abs(y.cpu().numpy().astype(np.float64) - x) <= 2.0 ** -11 * 3 * np.abs(x).max()).all()


def test_rows_beyond_2_to_the_31_elements():
    T, ld, heads, D = 2200, 1 << 20, 2, 128
    x, pos, tab, _ = case(T, heads, D, D, 1, False)
    big = torch.empty((T, ld), dtype=torch.float16, device="cuda")
    view = big.view(T, ld // D, D)[:, -heads:]
    view.copy_(torch.from_numpy(x))
    want = ref.turned(x, pos, tab)
    same(atom.atom_rotary(view, *gpu(pos, tab)), want)
    atom.atom_rotary(view, *gpu(pos, tab), out=view)
    same(view, want)


def test_captured_and_replayed_on_another_stream():
    x, pos, tab, axis = case(33, 12, 128, 128, 3, False)
    xd, pd, td = gpu(x, pos, tab)
    out = torch.zeros_like(xd)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        atom.atom_rotary(xd, pd, td, axis, out=out)
    for seed in range(3):
        y, p, _, _ = case(33, 12, 128, 128, 3, False, seed=seed)
        xd.copy_(torch.from_numpy(y))
        pd.copy_(torch.from_numpy(p))
        graph.replay()
        torch.cuda.synchronize()
        same(out, ref.turned(y, p, tab, axis))
    with torch.cuda.stream(stream):
        got = atom.atom_rotary(xd, pd, td, axis)
    stream.synchronize()
    assert torch.equal(got, out)


@pytest.mark.parametrize("T,heads,D,R,axes", [
    (1500, 5, 128, 128, 1), (903, 9, 80, 32, 3), (2049, 8, 64, 64, 2), (77, 71, 128, 64, 1), (7001, 29, 128, 128, 1), (6601, 30, 128, 96, 3)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_bits_of_many_heads_and_tokens(T, heads, D, R, axes, interleaved):
    """Four heads to a lane, the last lane's fewer; the largest past the caches."""
    x, pos, tab, axis = case(T, heads, D, R, axes, interleaved, seed=1)
    want = ref.turned(x, pos, tab, axis, interleaved, interleaved)
    xd, pd, td = gpu(x, pos, tab)
    same(atom.atom_rotary(xd, pd, td, axis, interleaved, interleaved), want)
    atom.atom_rotary(xd, pd, td, axis, interleaved, interleaved, out=xd)
    same(xd, want)
