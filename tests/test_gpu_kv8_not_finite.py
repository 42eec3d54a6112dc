"""Infinities and NaN in the paged 8-bit KV cache show: a block that takes one has a scale that is not finite from then on, and queries that see
such a block give NaN; nothing else changes."""
import numpy as np
import pytest
import torch

import paper_2310_19102_amd as atom
import _kv8_ref as ref
from test_gpu_kv8 import Case, caches, i32, npy

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


# ---------------------------------------------------------------- attention


# (H, Hkv, bs, past, new, extra, route): route as Case.route() gives it, and whether tiles have 32 rows
ROUTES = [
    (8, 2, 16, [100, 40], [3, 1], 1, lambda r: not r[1] and not r[2]),
    (8, 2, 64, [900, 2000, 70], [1, 1, 1], 3000, lambda r: r[1] and not r[2]),              # pieces and merge
    (16, 2, 32, [110, 300], [4, 3], 1 << 13, lambda r: r[1] and not r[2]),                  # tiles of 32 rows
    (16, 2, 16, [100, 30], [60, 70], 1 << 16, lambda r: r[2] and r[3]),                     # tiles of 128 rows, in pieces
    (64, 8, 64, [300, 20], [1200, 700], 1, lambda r: r[2] and not r[3]),                    # and whole
    (128, 1, 32, [1500], [500], 1, lambda r: r[2]),                                         # more than 1024 keys to a workgroup
    (64, 8, 32, [100, 4500, 4200], [400, 1, 2], 1, lambda r: r[0] and r[1] and r[2])]                       # single tokens beside tiles


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("what", ["k nan", "k inf", "v nan", "v inf", "k -inf"])
@pytest.mark.parametrize("H,Hkv,bs,past,new,extra,route", ROUTES, ids=range(len(ROUTES)))
def test_queries_that_see_a_spoiled_block_give_nan(H, Hkv, bs, past, new, extra, route, what, D):
    """Blocks at the beginning, in the middle and among the new tokens of a request, of its last cache head: exactly the queries that see a key of one, of that
    head, are NaN."""
    c = Case(H, Hkv, D, bs, past, new, seed=H + bs, extra=extra)
    assert route(c.route())
    group, clean = H // Hkv, c.call()
    side = c.kc if what[0] == "k" else c.vc
    b = 0                                                   # the request whose blocks are spoiled
    for j in sorted({0, past[b] // (2 * bs), (past[b] + new[b] // 2) // bs, (past[b] + new[b] - 1) // bs}, reverse=True):
        page = int(c.table[b, j])
        kept = side[1][page, Hkv - 1].clone()
        side[1][page, Hkv - 1] = float(what[2:])
        got = c.call()
        assert torch.equal(got[:, :H - group], clean[:, :H - group])
        sees = torch.zeros(c.T, dtype=torch.bool, device="cuda")
        sees[:new[b]] = past[b] + torch.arange(new[b], device="cuda") >= j * bs
        mine = got[:, H - group:]
        assert mine[sees].isnan().all() and mine[~sees].isfinite().all(), j
        # (a tile's other rows may move their weights' bound at other places: the last bits, and no more)
        assert ((mine[~sees].float() - clean[:, H - group:][~sees].float()).abs() <= 2.0 ** -9 * clean[:, H - group:][~sees].float().abs() + 1e-3).all()
        side[1][page, Hkv - 1] = kept
    assert torch.equal(c.call(), clean)


def test_an_overflow_in_a_step_shows_in_the_answer():
    """A NaN in one head's new key, from the append to the output: that request's later queries of that head, and no other."""
    H, Hkv, D, bs = 8, 2, 64, 16
    c = Case(H, Hkv, D, bs, [20, 33, 0], [2, 1, 40], seed=5)
    slot = torch.cat([c.table[b, (p + i) // bs][None] * bs + (p + i) % bs for b, (p, n) in enumerate(((20, 2), (33, 1), (0, 40))) for i in range(n)])
    k, v = (torch.randn((43, Hkv, D), generator=torch.Generator().manual_seed(3)).to(torch.float16).cuda() for _ in "kv")
    for x, at in ((k, (2, 1, 5)), (v, (3 + 20, 0, 9))):     # request 1's only token, request 2's twenty-first
        clean = x.clone()
        x[at] = float("nan")
        atom.atom_kv8_append(k, v, c.kc, c.vc, slot)
        got = c.call().view(43, Hkv, -1)
        want = torch.zeros((43, Hkv), dtype=torch.bool, device="cuda")
        if x is k:
            want[2, 1] = True
        else:
            want[3 + 16:, 0] = True                         # from the block's first row on: its scale is the block's
        assert torch.equal(got.isnan().all(2), want) and torch.equal(got.isnan().any(2), want)
        x.copy_(clean)
        c.kc[1].nan_to_num_(0.01)
