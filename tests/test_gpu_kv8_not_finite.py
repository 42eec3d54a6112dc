"""Infinities and NaN in the paged 8-bit KV cache show: a block that takes one has a scale that is not finite from then on; nothing else changes."""
import numpy as np
import pytest
import torch

import paper_2310_19102_amd as atom
import _kv8_ref as ref
from test_gpu_kv8 import caches, i32, npy

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- append


# NaN of every kind that fp16 has (signalling, quiet, negative, all bits), and both infinities
VALUES = [0x7c01, 0x7e00, 0xfe00, 0xffff, 0x7c00, 0xfc00]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bs,Hkv,T", [
    (16, 2, 45), (64, 2, 150), (128, 3, 200),               # a wavefront for a token and head
    (16, 40, 400), (32, 30, 500),                           # many tokens, a run to a wavefront
    (64, 3, 400), (128, 2, 700)])                           # and the four wavefronts of a workgroup on one run
def test_append_keeps_what_is_not_finite(D, bs, Hkv, T):
    """A run with a NaN makes its block's scale NaN and its own codes 0, older rows keep theirs; one with an infinity makes the scale infinite and all codes
    0; later rows change neither; the block's next first row does."""
    g = torch.Generator(device="cuda").manual_seed(bs + T)
    k, v = (torch.randn((T, Hkv, D), generator=g, device="cuda").to(torch.float16) for _ in "kv")
    first = 2 * bs + 5                                      # the first run stands behind five older rows
    blocks = (first + T) // bs + 3
    kc, vc = caches(blocks, Hkv, bs, D, seed=1)
    kc[1][2, 0] = 1e-4                                      # a scale that the rows' finite values would raise
    before = [(npy(c), npy(s)) for c, s in (kc, vc)]
    slot = torch.arange(first, first + T, dtype=torch.int32, device="cuda")
    want = [ref.append(npy(x), c, s, npy(slot)) for x, (c, s) in zip((k, v), before)]
    bad = [(1, 0, 3), (T - 1, Hkv - 1, D - 1), (bs + 2, 0, 0)]           # token, head, dimension: in the first block, the last one, one between
    for bits in VALUES:
        for (c, s), (c0, s0) in zip((kc, vc), before):
            c.copy_(torch.from_numpy(c0))
            s.copy_(torch.from_numpy(s0))
        x, y = k.clone(), v.clone()
        for t, h, d in bad:
            x.view(torch.int16)[t, h, d] = bits - 65536 if bits >= 32768 else bits
            y.view(torch.int16)[t, (h + 1) % Hkv, d] = bits - 65536 if bits >= 32768 else bits
        atom.atom_kv8_append(x, y, kc, vc, slot)
        nan = (bits & 0x3ff) != 0
        for side, ((codes, scale), (wc, ws), (c0, _)) in enumerate(zip((kc, vc), want, before)):
            wc, ws = wc.copy(), ws.copy()
            for t, h, d in bad:
                block, h = int(slot[t]) // bs, (h + side) % Hkv
                o, end = max(first - block * bs, 0), min(first + T - block * bs, bs)
                ws[block, h] = np.nan if nan else np.inf
                wc[block, h, :o] = c0[block, h, :o] if nan else 0
                wc[block, h, o:end] = 0
            assert np.array_equal(npy(scale), ws, equal_nan=True) and np.array_equal(npy(codes), wc), hex(bits)
        # one more row behind the last one, finite: its block stays as it is
        at = first + T
        block, row = divmod(at, bs)
        if row:
            scale = kc[1][block].clone()
            atom.atom_kv8_append(k[:1], v[:1], kc, vc, i32(at))
            assert torch.equal(kc[1][block].isfinite(), scale.isfinite()) and not kc[1][block, Hkv - 1].isfinite()
            assert (kc[0][block, Hkv - 1, row] == 0).all()
        # used again from its first row the block is like any other
        got = [(c[3:4].clone(), s[3:4].clone()) for c, s in (kc, vc)]
        assert not got[0][1][0, 0].isfinite()
        atom.atom_kv8_append(k[:7], v[:7], *got, torch.arange(7, dtype=torch.int32, device="cuda"))
        for xx, (c, s) in zip((k, v), got):
            wc, ws = ref.append(npy(xx[:7]), np.zeros((1, Hkv, bs, D), np.int8), np.zeros((1, Hkv), np.float32), np.arange(7))
            assert np.array_equal(npy(s), ws) and np.array_equal(npy(c[:, :, :7]), wc[:, :, :7])
