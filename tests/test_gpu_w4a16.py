"""Linear layers on 4-bit weights with fp16 activations, and the gated half of a feed-forward block, against the definition in
64 bits with the error that the library's arithmetic may have."""
import numpy as np
import pytest
import torch

import _fp16_layer_ref as ref
import paper_2310_19102_amd as atom

pytestmark = pytest.mark.gpu


def weights(N, K, O, rng):
    scale = (0.01 * (1 + 0.2 * rng.standard_normal((N, K // 128)))).astype(np.float16)
    return (rng.integers(0, 256, (N, (K - O) // 2)).astype(np.uint8), rng.integers(-128, 128, (N, O)).astype(np.int8), scale)


def case(M, N, K, O=128, matrices=1, seed=0):
    rng = np.random.default_rng([M, N, K, O, seed])
    x = (rng.standard_normal((M, K)) * np.exp(rng.standard_normal(K))).astype(np.float16)
    gamma = (1 + 0.1 * rng.standard_normal(K)).astype(np.float16)
    return x, gamma, rng.permutation(K).astype(np.int32), [weights(N, K, O, rng) for _ in range(matrices)], rng


def gpu(a):
    return None if a is None else tuple(gpu(x) for x in a) if isinstance(a, tuple) else torch.from_numpy(a).cuda()


def close(got, want, tol, what=""):
    got = got.cpu().numpy().astype(np.float64)
    assert np.isfinite(want).all() and got.shape == want.shape
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, first {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]} within {tol[bad][0]}"


SIZES = [(1, 1, 256, 128), (1, 16, 256, 128), (2, 17, 384, 128), (1, 4097, 4096, 128), (3, 100, 512, 256), (5, 33, 640, 384), (8, 129, 1280, 128),
         (15, 31, 1152, 128), (16, 48, 1024, 128), (17, 64, 1024, 128), (31, 15, 2048, 128), (32, 500, 768, 128), (33, 77, 4224, 128), (48, 65, 1664, 256),
         (63, 40, 1408, 128), (64, 260, 896, 128), (65, 130, 1024, 128), (130, 90, 512, 128), (300, 70, 640, 128), (1, 300, 32768, 128), (4, 96, 11008, 128),
         (1, 20000, 512, 128), (7, 9001, 384, 128), (40, 3000, 2176, 128)]


@pytest.mark.parametrize("M,N,K,O", SIZES)
@pytest.mark.parametrize("norm,index,add", [(True, True, False), (False, False, True), (False, True, True), (True, False, False)])
def test_linear(M, N, K, O, norm, index, add):
    x, gamma, idx, (w,), rng = case(M, N, K, O)
    gamma, idx = gamma if norm else None, idx if index else None
    residual = rng.standard_normal((M, N)).astype(np.float16) if add else None
    want, tol = ref.linear(x, gamma, 1e-5, idx, w, residual)
    args = (gpu(x), gpu(gamma), 1e-5, gpu(idx), *gpu(w), gpu(residual))
    y = atom.atom_w4a16_linear(*args)
    close(y, want, tol, "linear")
    again = atom.atom_w4a16_linear(*args)
    assert torch.equal(y, again)                              # the order of the sums depends on the sizes alone


@pytest.mark.parametrize("M,N,K,O", SIZES)
@pytest.mark.parametrize("norm,index", [(True, True), (False, False), (False, True)])
def test_swiglu(M, N, K, O, norm, index):
    x, gamma, idx, (gate, up), _ = case(M, N, K, O, 2)
    x, gamma, idx = x * np.float16(0.25), gamma if norm else None, idx if index else None
    want, tol = ref.swiglu(x, gamma, 1e-5, idx, gate, up)
    fits = np.abs(want) < 60000
    want, tol = np.where(fits, want, 0), np.where(fits, tol, np.inf)
    h = atom.atom_w4a16_swiglu(gpu(x), gpu(gamma), 1e-5, gpu(idx), gpu(gate), gpu(up))
    close(torch.where(torch.from_numpy(fits).cuda(), h, 0.0), want, tol, "swiglu")


@pytest.mark.parametrize("M", [1, 6, 20, 64, 100])
def test_strides_and_memory_of_the_callers(M):
    N, K = 70, 768
    x, gamma, idx, (w,), rng = case(M, N, K)
    residual = rng.standard_normal((M, N)).astype(np.float16)
    want, tol = ref.linear(x, gamma, 1e-5, idx, w, residual)
    wide = torch.full((M, K + 24), 9.0, dtype=torch.float16, device="cuda")
    wide[:, 8:8 + K] = gpu(x)
    out = torch.full((M + 1, N + 5), 3.0, dtype=torch.float16, device="cuda")
    view = out[:M, 2:2 + N]
    view.copy_(gpu(residual))                                 # in place on the residual
    work = torch.full((atom.atom_w4a16_workspace_bytes(M, N, K) + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    y = atom.atom_w4a16_linear(wide[:, 8:8 + K], gpu(gamma), 1e-5, gpu(idx), *gpu(w), view, out=view, workspace=work[:-512])
    assert y is view
    close(view, want, tol)
    assert bool((out[M:] == 3).all()) and bool((out[:, :2] == 3).all()) and bool((out[:, 2 + N:] == 3).all())
    assert bool((work[-512:] == 0x5A).all())


def test_three_bit_weights_and_those_of_the_library():
    """Weights as atom_quantize_weight gives them, in 4 and in 3 bits, and the layer that the paper's W4A4 path computes from them."""
    M, N, K = 9, 200, 1024
    x, gamma, idx, _, rng = case(M, N, K)
    w16 = (0.05 * rng.standard_normal((N, K))).astype(np.float16)
    for bits in (4, 3):
        w = atom.atom_quantize_weight(gpu(w16), gpu(idx), bits=bits)
        want, tol = ref.linear(x, gamma, 1e-5, idx, tuple(t.cpu().numpy() for t in w))
        close(atom.atom_w4a16_linear(gpu(x), gpu(gamma), 1e-5, gpu(idx), *w), want, tol, f"{bits} bits")


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("M", [3, 40])
def test_rows_keep_to_themselves(M, norm):
    """Rows of zeros, of what is not finite, of the largest and smallest numbers: nothing reaches another row."""
    N, K = 50, 640
    x, gamma, idx, (w,), _ = case(M, N, K)
    gamma = gamma if norm else None
    x[1] = 0
    clean, tol = ref.linear(x, gamma, 1e-5, idx, w)
    x[0, 7], x[M - 1, 100] = np.inf, np.nan
    y = atom.atom_w4a16_linear(gpu(x), gpu(gamma), 1e-5, gpu(idx), *gpu(w))
    rows = [m for m in range(M) if m not in (0, M - 1)]
    close(y[rows], clean[rows], tol[rows])
    got = y.cpu().numpy()
    assert (got[1] == 0).all() and np.isnan(got[M - 1]).all()
    if norm:
        assert np.isnan(got[0]).all()                         # infinity times the reciprocal root 0
    else:
        code = ref.codes_of(w[0], w[1])[:, list(idx).index(7)]
        assert np.array_equal(np.isnan(got[0]), code == 0) and np.array_equal(got[0][code != 0], np.where(code > 0, np.inf, -np.inf)[code != 0])
    x[0], x[M - 1] = 65504, 6e-8
    want, tol = ref.linear(x, gamma, 1e-5, idx, w)
    got = atom.atom_w4a16_linear(gpu(x), gpu(gamma), 1e-5, gpu(idx), *gpu(w))
    over = np.abs(want) > 65520 + tol
    assert np.array_equal(np.isinf(got.cpu().numpy())[over], np.ones(over.sum(), bool))
    sure = np.abs(want) < 65504 - tol
    close(torch.where(torch.from_numpy(sure).cuda(), got, 0.0), np.where(sure, want, 0), np.where(sure, tol, np.inf))


@pytest.mark.parametrize("M", [2, 20, 60])
def test_numbers_below_the_normal_ones_count(M):
    """fp16's smallest numbers times large scales: nothing is flushed on the way."""
    N, K = 33, 384
    x, _, idx, (w,), rng = case(M, N, K)
    x = (rng.integers(-40, 41, (M, K)) * 2.0 ** -24).astype(np.float16)
    w = (w[0], w[1], np.full_like(w[2], 2048))
    want, tol = ref.linear(x, None, 0.0, idx, w)
    assert np.abs(want).mean() > 0.05
    close(atom.atom_w4a16_linear(gpu(x), None, 0.0, gpu(idx), *gpu(w)), want, tol)


def test_gate_far_from_zero():
    """silu of very negative gates is 0 (or below fp16), of very positive ones the gate itself."""
    M, N, K = 2, 32, 256
    x, _, _, (gate, up), _ = case(M, N, K, matrices=2)
    x[:] = 0
    x[0, 0], x[1, 0] = 300, -300
    gate = (np.full_like(gate[0], 0x11), gate[1], np.full_like(gate[2], 0.5))
    up = (np.full_like(up[0], 0x22), up[1], np.full_like(up[2], 0.25))
    h = atom.atom_w4a16_swiglu(gpu(x), None, 0.0, None, gpu(gate), gpu(up)).cpu().numpy()
    assert (h[0] == 150 * 150).all() and (h[1] == 0).all()


def test_each_output_channel_and_group_counts_once():
    """One channel at a time: y is code times scale, exactly."""
    N, K, O = 40, 512, 128
    _, _, idx, (w,), _ = case(1, N, K, O)
    code = ref.codes_of(w[0], w[1])
    x = np.zeros((K, K), np.float16)
    x[np.arange(K), idx] = 1
    y = atom.atom_w4a16_linear(gpu(x), None, 0.0, gpu(idx), *gpu(w)).cpu().numpy()
    want = (code * np.repeat(w[2].astype(np.float64), 128, 1)).T.astype(np.float16)
    assert np.array_equal(y, want)
    for m in (0, 200, 511):                                   # a row alone takes another kernel's way
        y = atom.atom_w4a16_linear(gpu(x[m:m + 1].copy()), None, 0.0, gpu(idx), *gpu(w)).cpu().numpy()
        assert np.array_equal(y, want[m:m + 1])


def test_empty_calls():
    x, gamma, idx, (w, u), _ = case(4, 20, 512, matrices=2)
    none = torch.empty((0, 512), dtype=torch.float16, device="cuda")
    assert atom.atom_w4a16_linear(none, gpu(gamma), 1e-5, gpu(idx), *gpu(w)).shape == (0, 20)
    assert atom.atom_w4a16_swiglu(none, None, 1e-5, None, gpu(w), gpu(u)).shape == (0, 20)
    w = tuple(a[:0] for a in w)
    assert atom.atom_w4a16_linear(gpu(x), gpu(gamma), 1e-5, gpu(idx), *gpu(w)).shape == (4, 0)


@pytest.mark.parametrize("M", [1, 12, 50])
def test_two_graphs_that_share_a_workspace(M):
    N, K = 300, 1024
    x, gamma, idx, (w, u), _ = case(M, N, K, matrices=2)
    xd, gd, idd, wd, ud = gpu(x), gpu(gamma), gpu(idx), gpu(w), gpu(u)
    need = max(atom.atom_w4a16_workspace_bytes(M, N, K, gated=g) for g in (False, True))
    work = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    y, h = (torch.zeros((M, N), dtype=torch.float16, device="cuda") for _ in range(2))
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    with torch.cuda.graph(graphs[0]):
        atom.atom_w4a16_linear(xd, gd, 1e-5, idd, *wd, out=y, workspace=work)
    with torch.cuda.graph(graphs[1]):
        atom.atom_w4a16_swiglu(xd, gd, 1e-5, idd, wd, ud, out=h, workspace=work)
    for seed in range(3):
        xd.copy_(gpu(case(M, N, K, seed=seed)[0]))
        for g in (0, 1, 1, 0):
            graphs[g].replay()
        torch.cuda.synchronize()
        assert torch.equal(y, atom.atom_w4a16_linear(xd, gd, 1e-5, idd, *wd))
        assert torch.equal(h, atom.atom_w4a16_swiglu(xd, gd, 1e-5, idd, wd, ud))


def test_on_a_stream_of_the_callers():
    x, gamma, idx, (w,), _ = case(8, 500, 2048)
    args = (gpu(x), gpu(gamma), 1e-5, gpu(idx), *gpu(w))
    want = atom.atom_w4a16_linear(*args)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        y = atom.atom_w4a16_linear(*args)
    stream.synchronize()
    assert torch.equal(y, want)


def device_weights(N, K, O, g):
    r = lambda lo, hi, n, t: torch.randint(lo, hi, (N, n), generator=g, device="cuda", dtype=t)         # noqa: E731
    scale = (0.01 * (1 + 0.2 * torch.rand((N, K // 128), generator=g, device="cuda"))).to(torch.float16)
    return r(0, 256, (K - O) // 2, torch.uint8), r(-128, 128, O, torch.int8), scale


@pytest.mark.parametrize("M,gated,norm", [(20, False, True), (40, True, False), (33, True, True), (64, False, False)])
def test_many_outputs_whole_rows_of_scales_in_turn(M, gated, norm):
    """So many outputs that no workgroup shares its K channels: 80 groups of scales, which come 64 at a time.  Every hundredth output
    and the last ones against 64 bits."""
    K, O, N = 10240, 256, 25607 if gated else 51195
    g = torch.Generator(device="cuda").manual_seed(M)
    w = [device_weights(N, K, O, g) for _ in range(2 if gated else 1)]
    x, gamma, idx, _, _ = case(M, 1, K, O)
    x, gamma = x * np.float16(0.125 if gated else 1), gamma if norm else None
    some = np.unique(np.concatenate([np.arange(0, N, 101), np.arange(N - 140, N)]))
    few = [tuple(t[torch.from_numpy(some).cuda()].cpu().numpy() for t in m) for m in w]
    args = (gpu(x), gpu(gamma), 1e-5, gpu(idx))
    if gated:
        want, tol = ref.swiglu(x, gamma, 1e-5, idx, *few)
        got = atom.atom_w4a16_swiglu(*args, *w)
    else:
        want, tol = ref.linear(x, gamma, 1e-5, idx, *few)
        got = atom.atom_w4a16_linear(*args, *w[0])
    fits = np.abs(want) < 60000
    got = torch.where(torch.from_numpy(fits).cuda(), got[:, torch.from_numpy(some).cuda()], 0.0)
    close(got, np.where(fits, want, 0), np.where(fits, tol, np.inf))


@pytest.mark.parametrize("M", [1, 3, 8, 9, 16, 24, 50])
@pytest.mark.parametrize("K,O", [(1280, 1152), (2048, 640), (9088, 128), (4224, 4096)])
def test_many_outliers_and_few_groups(M, K, O):
    N = 50
    x, gamma, idx, (w, u), _ = case(M, N, K, O, 2)
    w, u = ((q4, q8, (s * np.float16(0.125)).astype(np.float16)) for q4, q8, s in (w, u))
    want, tol = ref.linear(x, gamma, 1e-5, idx, w)
    close(atom.atom_w4a16_linear(gpu(x), gpu(gamma), 1e-5, gpu(idx), *gpu(w)), want, tol)
    x = x * np.float16(0.125)
    want, tol = ref.swiglu(x, None, 1e-5, idx, w, u)
    fits = np.abs(want) < 60000
    got = atom.atom_w4a16_swiglu(gpu(x), None, 1e-5, gpu(idx), gpu(w), gpu(u))
    close(torch.where(torch.from_numpy(fits).cuda(), got, 0.0), np.where(fits, want, 0), np.where(fits, tol, np.inf))


@pytest.mark.parametrize("M", [1, 12, 20])
def test_a_normed_value_beyond_fp16_counts_as_infinite(M):
    N, K = 20, 512
    x, gamma, idx, (w,), _ = case(M, N, K)
    x[:] = 0
    x[:, 5], gamma[5] = 100, 60000                            # sqrt(512) * 60000
    y = atom.atom_w4a16_linear(gpu(x), gpu(gamma), 0.0, gpu(idx), *gpu(w)).cpu().numpy()
    code = ref.codes_of(w[0], w[1])[:, list(idx).index(5)]
    want = np.where(code == 0, np.nan, np.where(code > 0, np.inf, -np.inf)).astype(np.float16)
    assert np.array_equal(y, np.broadcast_to(want, y.shape), equal_nan=True)
