"""Linear and gated layers of up to 16 rows with so many outputs that a workgroup has two or four tiles of 16 channels, or several in turn, none of them laying out its
activations itself.  Sampled outputs, among them every place in a workgroup's tiles and the last ones, against 64 bits."""
import numpy as np
import pytest
import torch

import _fp16_layer_ref as ref
import paper_2310_19102_amd as atom
from test_gpu_w4a16 import case, close, device_weights, gpu

pytestmark = pytest.mark.gpu

# no N is a multiple of a tile; from 33001 on workgroups have a second tile
SIZES = [(8, 12289, 4096), (8, 8003, 8192), (16, 20003, 8192), (12, 28675, 4096), (6, 9001, 8192), (16, 8003, 8192), (9, 40001, 4096), (8, 40001, 4096), (10, 9001, 640)]
WAYS = [(True, True, False), (False, False, True), (False, True, False), (True, False, True)]      # norm, index, residual


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("norm,index,add", WAYS)
@pytest.mark.parametrize("gated", [False, True])
def test_sampled_outputs(M, N, K, norm, index, add, gated):
    O = 128
    g = torch.Generator(device="cuda").manual_seed(M + N)
    w = [device_weights(N, K, O, g) for _ in range(2 if gated else 1)]
    x, gamma, idx, _, rng = case(M, 1, K, O)
    x, gamma, idx = x * np.float16(0.125 if gated else 1), gamma if norm else None, idx if index else None
    some = np.unique(np.concatenate([np.arange(0, 130), np.arange(131, N, 61), np.arange(N - 140, N)]))
    at = torch.from_numpy(some).cuda()
    few = [tuple(t[at].cpu().numpy() for t in m) for m in w]
    args = (gpu(x), gpu(gamma), 1e-5, gpu(idx))
    out = torch.full((M + 1, N), 7.0, dtype=torch.float16, device="cuda")
    if gated:
        want, tol = ref.swiglu(x, gamma, 1e-5, idx, *few)
        got = atom.atom_w4a16_swiglu(*args, *w, out=out[:M])
        again = atom.atom_w4a16_swiglu(*args, *w)
    else:
        residual = gpu(rng.standard_normal((M, N)).astype(np.float16)) if add else None
        want, tol = ref.linear(x, gamma, 1e-5, idx, *few, residual[:, at].cpu().numpy() if add else None)
        got = atom.atom_w4a16_linear(*args, *w[0], residual, out=out[:M])
        again = atom.atom_w4a16_linear(*args, *w[0], residual)
    assert bool((out[M] == 7).all())
    fits = np.abs(want) < 60000
    assert fits.mean() > 0.9
    close(torch.where(torch.from_numpy(fits).cuda(), got[:, at], 0.0), np.where(fits, want, 0), np.where(fits, tol, np.inf))
    assert torch.equal(got.view(torch.int16), again.view(torch.int16))
