"""The rotary append where a workgroup has several cache heads, and a lane several times four query heads, in turn: bit for bit, as in test_gpu_rotary_kv8.py."""
import numpy as np
import pytest
import torch

import _fp16_layer_ref as ref
import _kv8_ref as kv8
import paper_2310_19102_amd as atom
from test_gpu_rotary_kv8 import check, run, step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,Hkv,D,bs,axes,interleaved", [
    (256, 32, 128, 16, 1, False), (256, 32, 128, 64, 3, True), (256, 32, 64, 128, 1, False),                   # two heads a workgroup
    (8192, 5, 128, 16, 1, True), (2040, 32, 64, 32, 2, False),                                                # four (and a remainder)
    (8192, 9, 64, 16, 1, False)])                                                                              # eight
def test_single_tokens(n, Hkv, D, bs, axes, interleaved):
    """Zeros, large rows, scales that grow under older rows, tokens without a slot, and rows that are not finite, in every head."""
    s = step([(i * 7 % (3 * bs), 1) for i in range(n)] if n < 1000 else [(i % 7, 1) for i in range(n)], 1, Hkv, D, bs, D // 2, axes, padding=5, missing=range(3, n, 11))
    s["qkv"][5] = 0
    s["qkv"][6, 1::2] *= 300
    s["qkv"][40:60, 2::3] *= 0.001
    s["k"][1][:] *= 0.5
    check(s, run(s, interleaved), interleaved)
    k = s["qkv"][:, 1:1 + Hkv]
    k[7, :, 3], k[8, Hkv - 1, D - 1], k[12, 0, 0] = np.nan, np.inf, -np.inf
    _, kc, vc, _ = run(s, interleaved)
    with np.errstate(invalid="ignore"):
        want = ref.turned(s["qkv"][:, :1 + Hkv], s["pos"], s["tab"], s["axis"], interleaved)[:, 1:]
        codes, scale = kv8.append(np.where(np.isfinite(want), want, 0), *s["k"], s["slot"])
    spoilt = np.zeros(scale.shape, bool)
    for t in (7, 8, 12):
        spoilt[s["slot"][t] // bs] = ~np.isfinite(want[t]).all(1)
    assert spoilt.sum() == Hkv + 2
    got = kc[1].cpu().numpy()
    assert np.array_equal(~np.isfinite(got), spoilt) and np.array_equal(got[~spoilt], scale[~spoilt])
    assert np.array_equal(kc[0].cpu().numpy()[~spoilt], codes[~spoilt])


@pytest.mark.parametrize("pairs,Hkv,bs,axes,interleaved", [
    ([(0, 2500), (70, 1990), (3, 1)], 20, 64, 1, False), ([(0, 2500), (70, 1990), (3, 1)], 20, 128, 3, True),  # two heads a workgroup
    ([(100, 4000), (0, 1), (0, 4097)], 5, 16, 1, True),                                                       # four, short blocks
    ([(33, 9000), (5, 3), (0, 7370)], 9, 64, 1, False), ([(33, 9000), (5, 3), (0, 7370)], 9, 128, 1, True)])    # eight
def test_prompts(pairs, Hkv, bs, axes, interleaved):
    s = step(pairs, 1, Hkv, 128, bs, 64, axes, padding=30)
    s["qkv"][200:230, 3:] *= 50
    check(s, run(s, interleaved), interleaved)


@pytest.mark.parametrize("pairs,H,Hkv,D,axes,interleaved", [
    ([(0, 1300), (9, 1)], 64, 2, 128, 1, False), ([(5, 2800)], 20, 2, 128, 3, True), ([(0, 4200)], 13, 1, 128, 1, True), ([(0, 2900), (7, 300)], 45, 1, 64, 2, False)])
def test_queries(pairs, H, Hkv, D, axes, interleaved):
    """Eight heads to a lane, the last lane's fewer; in place too."""
    s = step(pairs, H, Hkv, D, 64, D, axes)
    check(s, run(s, interleaved), interleaved)
    got = run(s, interleaved, out="q")
    check(s, got, interleaved)
    assert np.array_equal(got[3][:, H:].cpu().numpy(), s["qkv"][:, H:])
