"""Single tokens, step after step, into blocks whose scales grow under their older rows: every number of older rows, in some or in all heads of a step, bit for bit
as in test_gpu_rotary_kv8.py."""
import numpy as np
import pytest
import torch

import _fp16_layer_ref as ref
import _kv8_ref as kv8
import paper_2310_19102_amd as atom

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,bs,Hkv,n,axes,interleaved", [
    (128, 128, 2, 19, 1, False), (64, 128, 3, 17, 2, True), (128, 64, 3, 40, 3, True), (64, 64, 5, 16, 1, False), (128, 32, 2, 33, 1, True), (64, 16, 4, 50, 1, False),
    (128, 64, 32, 256, 1, False), (128, 64, 2, 5, 1, False), (64, 128, 2, 3, 1, True)])
def test_every_number_of_older_rows(D, bs, Hkv, n, axes, interleaved):
    """Requests a few rows apart, so that a step meets many of them; a row grows with a chance of a half, so some wavefronts have one such row and others all."""
    rng = np.random.default_rng([D, bs, Hkv, n])
    steps = bs + 3 if n < 100 else 12
    ids = rng.permutation(3 * n)
    first = rng.integers(0, bs, n) if n >= 100 else np.arange(n) * 3 % bs
    tab = ref.table(3 * bs, D // 4)
    axis = None if axes == 1 else rng.integers(0, axes, D // 4).tolist()
    sides = [(rng.integers(-127, 128, (3 * n, Hkv, bs, D)).astype(np.int8), np.full((3 * n, Hkv), 0.004, np.float32)) for _ in range(2)]
    caches = [tuple(torch.from_numpy(a.copy()).cuda() for a in side) for side in sides]
    tabd = torch.from_numpy(tab).cuda()
    grown = 0
    for i in range(steps):
        at = first + i
        slot = (ids[3 * np.arange(n) + at // bs] * bs + at % bs).astype(np.int32)
        slot[rng.random(n) < 0.1] = -1
        size = np.where(rng.random((n, 2 * Hkv, 1)) < 0.5, 1.02 ** i, 0.5)
        rows = np.clip(rng.standard_normal((n, 2 * Hkv, D)) * size, -30000, 30000).astype(np.float16)
        pos = at.astype(np.int32) if axes == 1 else np.stack([at] + [rng.integers(0, 3 * bs, n) for _ in range(axes - 1)]).astype(np.int32)
        turned = ref.turned(rows[:, :Hkv], pos, tab, axis, interleaved)
        new = []
        for x, side in ((turned, sides[0]), (rows[:, Hkv:], sides[1])):
            new.append(kv8.append(x, *side, slot))
            older = slot[slot >= 0] // bs
            grown += (new[-1][1][older] > side[1][older]).sum()
        rd = torch.from_numpy(rows).cuda()
        atom.atom_rotary_kv8_append(None, rd[:, :Hkv], rd[:, Hkv:], *caches, torch.from_numpy(slot).cuda(), torch.from_numpy(pos).cuda(), tabd, axis, interleaved)
        for cache, (codes, scale) in zip(caches, new):
            assert np.array_equal(cache[1].cpu().numpy().view(np.uint32), scale.view(np.uint32)), i
            assert np.array_equal(cache[0].cpu().numpy(), codes), i
        sides = new
    assert grown > n * Hkv
