"""Queries turned, keys turned and appended to the paged 8-bit cache, values appended: codes, scales and queries bit for bit
against IEEE fp32 steps in numpy."""
import numpy as np
import pytest
import torch

import _fp16_layer_ref as ref
import _kv8_ref as kv8
import paper_2310_19102_amd as atom

pytestmark = pytest.mark.gpu


def step(pairs, H, Hkv, D, bs, R=None, axes=1, seed=0, padding=0, missing=()):
    """A step of requests with (past, new) tokens: rows as slices of one projection, caches in use, slots of blocks in a random
    order; `padding` tokens without a slot at the end, and those in `missing` without one between."""
    R = R or D
    rng = np.random.default_rng([seed, H, Hkv, D, bs, len(pairs)])
    need = [-(-(p + n) // bs) for p, n in pairs]
    ids, at, slot, pos = rng.permutation(sum(need) + 3), 0, [], []
    for (p, n), blocks in zip(pairs, need):
        mine = ids[at:at + blocks]
        at += blocks
        for i in range(p, p + n):
            slot.append(mine[i // bs] * bs + i % bs)
            pos.append(i)
    slot = np.array(slot + [-1] * padding, np.int32)
    slot[list(missing)] = -1
    T = len(slot)
    P = max(pos + [0]) + 1
    pos = np.array(pos + [0] * padding, np.int32)
    if axes > 1:
        pos = np.stack([pos] + [rng.integers(0, P, T).astype(np.int32) for _ in range(axes - 1)])
    s = {"qkv": rng.standard_normal((T, H + 2 * Hkv, D)).astype(np.float16), "slot": slot, "pos": pos, "tab": ref.table(P, R // 2),
         "axis": None if axes == 1 else rng.integers(0, axes, R // 2).tolist(), "H": H, "Hkv": Hkv}
    n = sum(need) + 3
    for side in "kv":
        s[side] = (rng.integers(-127, 128, (n, Hkv, bs, D)).astype(np.int8), (rng.random((n, Hkv)) * 0.04).astype(np.float32))
    return s


def run(s, interleaved=False, out=None, queries=True):
    H, Hkv = s["H"], s["Hkv"]
    qkv = torch.from_numpy(s["qkv"]).cuda()
    caches = [tuple(torch.from_numpy(a.copy()).cuda() for a in s[side]) for side in "kv"]
    q, kc, vc = atom.atom_rotary_kv8_append(qkv[:, :H] if queries else None, qkv[:, H:H + Hkv], qkv[:, H + Hkv:], *caches,
                                            *(torch.from_numpy(s[x]).cuda() for x in ("slot", "pos", "tab")), s["axis"], interleaved,
                                            out=qkv[:, :H] if out == "q" else out)
    assert kc[0] is caches[0][0] and vc[1] is caches[1][1]
    torch.cuda.synchronize()
    return q, kc, vc, qkv


def check(s, got, interleaved=False, queries=True):
    H, Hkv = s["H"], s["Hkv"]
    q, kc, vc, _ = got
    with np.errstate(invalid="ignore"):
        turned = ref.turned(s["qkv"][:, :H + Hkv], s["pos"], s["tab"], s["axis"], interleaved)
    if queries:
        assert np.array_equal(q.cpu().numpy().view(np.uint16), turned[:, :H].astype(np.float16).view(np.uint16))
    for rows, side, cache in ((turned[:, H:], "k", kc), (s["qkv"][:, H + Hkv:], "v", vc)):
        codes, scale = kv8.append(rows, *s[side], s["slot"])
        assert np.array_equal(cache[1].cpu().numpy().view(np.uint32), scale.view(np.uint32)), side
        assert np.array_equal(cache[0].cpu().numpy(), codes), side


REQUESTS = {"one": [(0, 1)], "decode": [(17, 1), (15, 1), (16, 1), (0, 1), (63, 1), (127, 1), (128, 1)], "short": [(3, 5), (0, 17), (30, 2), (5, 1)],
            "mixed": [(100, 1), (9, 150), (64, 1), (0, 33)], "prompt": [(0, 300)], "prompts": [(0, 257), (120, 140), (7, 1)],
            "batch": [(i * 5 % 77, 1) for i in range(300)], "large": [(50, 700), (0, 1), (1, 513)]}


@pytest.mark.parametrize("requests", REQUESTS)
@pytest.mark.parametrize("H,Hkv,D,bs,R,axes,interleaved", [
    (4, 4, 128, 64, 128, 1, False), (16, 2, 128, 16, 128, 3, False), (5, 1, 64, 128, 64, 1, True), (8, 8, 64, 32, 16, 4, False), (12, 12, 128, 128, 64, 2, True)])
def test_bits(requests, H, Hkv, D, bs, R, axes, interleaved):
    s = step(REQUESTS[requests], H, Hkv, D, bs, R, axes)
    got = run(s, interleaved)
    check(s, got, interleaved)
    assert np.array_equal(got[3].cpu().numpy(), s["qkv"])     # the projection's output is left as it was


@pytest.mark.parametrize("requests", ["one", "short", "prompts"])
def test_queries_in_place_and_without_queries(requests):
    s = step(REQUESTS[requests], 8, 2, 128, 32)
    got = run(s, out="q")
    check(s, got)
    assert np.array_equal(got[3][:, 8:].cpu().numpy(), s["qkv"][:, 8:])
    got = run(s, queries=False)
    assert got[0] is None
    check(s, got, queries=False)


@pytest.mark.parametrize("requests,missing", [("short", [0, 9, 24]), ("prompt", [0, 64, 65, 130, 299]), ("batch", [5, 6, 200])])
def test_padding_and_tokens_without_a_slot(requests, missing):
    """They write nothing; a hole in a block begins another run behind it, which is another block here."""
    s = step(REQUESTS[requests], 4, 2, 64, 16, padding=70)
    bs = 16
    if requests == "prompt":                                  # whole blocks out: what follows a hole begins a block
        for m in missing:
            s["slot"][m // bs * bs:(m // bs + 1) * bs] = -1
    elif requests == "short":                                 # the first tokens of their runs out
        s["slot"][[0, 5]] = -1
    else:
        s["slot"][missing] = -1
    s["slot"][-1], s["slot"][-5] = s["k"][0].shape[0] * bs, 2 ** 31 - 1     # outside the cache
    check(s, run(s))


def test_twice_is_once():
    s = step(REQUESTS["mixed"], 4, 2, 128, 32)
    q, kc, vc, qkv = run(s)
    before = [t.clone() for t in (q, *kc, *vc)]
    q, kc, vc = atom.atom_rotary_kv8_append(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], kc, vc, *(torch.from_numpy(s[x]).cuda() for x in ("slot", "pos", "tab")))
    assert all(torch.equal(a, b) for a, b in zip(before, (q, *kc, *vc)))


def test_zero_rows_large_rows_and_grown_scales():
    s = step([(20, 12), (40, 3), (0, 64), (10, 1)], 2, 2, 128, 64)
    s["qkv"][:12] *= 200                                      # scales that grow under older rows
    s["qkv"][12:15] = 0                                       # nothing new: the scale stays
    s["qkv"][15:79, :, :64] = 60000                           # turned sums beyond fp16's range
    s["qkv"][15:79, :, 64:] = -60000
    s["k"][1][:] = 0.01
    check(s, run(s)[:3] + (None,), queries=False)


def test_what_is_not_finite_stays_in_its_block_and_head():
    s = step([(5, 20), (70, 1), (0, 90)], 3, 3, 64, 32)
    s["qkv"][4, 4, 7] = np.nan                                # a key of head 1
    s["qkv"][22, 3, 60] = np.inf                              # a key of head 0
    s["pos"][30] = 10 ** 6                                    # outside the table: the keys of all heads
    q, kc, vc, _ = run(s)
    want = ref.turned(s["qkv"][:, :6], s["pos"], s["tab"])
    bad = s["slot"][[4, 22, 30]] // 32
    scale = kc[1].cpu().numpy()
    with np.errstate(invalid="ignore"):
        codes, scales = kv8.append(np.nan_to_num(want[:, 3:], nan=0, posinf=0, neginf=0), *s["k"], s["slot"])
    touched = np.zeros(scale.shape, bool)
    touched[bad[0], 1] = touched[bad[1], 0] = touched[bad[2]] = True
    assert np.array_equal(~np.isfinite(scale), touched)
    assert np.array_equal(scale[~touched], scales[~touched])
    assert np.array_equal(kc[0].cpu().numpy()[~touched], codes[~touched])
    for block, head, rows in ((bad[0], 1, [4]), (bad[2], 2, [30])):           # codes under such a scale are 0
        run_rows = s["slot"][(s["slot"] // 32 == block)] % 32
        assert (kc[0].cpu().numpy()[block, head, run_rows] == 0).all()
    assert np.isfinite(vc[1].cpu().numpy()).all()
    got = q.cpu().numpy()
    assert np.isnan(got[30]).all() and np.array_equal(np.isnan(got), np.isnan(want[:, :3]))


def test_captured_with_new_lengths_on_every_replay():
    s = step([(30, 1)] * 9, 8, 2, 128, 16, padding=3)
    H, Hkv = 8, 2
    qkv = torch.from_numpy(s["qkv"]).cuda()
    slot, pos, tab = (torch.from_numpy(s[x]).cuda() for x in ("slot", "pos", "tab"))
    caches = [tuple(torch.from_numpy(a.copy()).cuda() for a in s[side]) for side in "kv"]
    out, graph = torch.zeros((12, H, 128), dtype=torch.float16, device="cuda"), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        atom.atom_rotary_kv8_append(qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:], *caches, slot, pos, tab, out=out)
    for seed in range(4):
        t = step([(9 + 3 * seed, 1)] * 9, 8, 2, 128, 16, padding=3, seed=seed + 1)
        n = min(len(t["k"][0]), len(caches[0][0]))
        t["slot"] = np.where(t["slot"] < n * 16, t["slot"], -1).astype(np.int32)
        t["tab"] = s["tab"]
        for dst, src in ((qkv, "qkv"), (slot, "slot"), (pos, "pos")):
            dst.copy_(torch.from_numpy(t[src]))
        for cache, side in zip(caches, "kv"):
            t[side] = tuple(a.cpu().numpy() for a in cache)
        graph.replay()
        torch.cuda.synchronize()
        check(t, (out, *caches, None))


@pytest.mark.parametrize("bs", [16, 32, 64, 128])
@pytest.mark.parametrize("axes,interleaved,padding", [(1, False, 0), (3, True, 100)])
def test_bits_of_many_tokens_and_several_heads_to_a_workgroup(bs, axes, interleaved, padding):
    s = step([(0, 2100), (37, 1000), (9, 1), (501, 1111), (0, 2)], 4, 16, 64, bs, 32, axes, padding=padding)
    s["slot"][1500:1500 + bs] = -1                            # a hole of a block's length
    if bs > 16:
        s["slot"][1500 // bs * bs:1500 // bs * bs + bs] = -1  # (and what began the block before it)
    check(s, run(s, interleaved), interleaved)


@pytest.mark.parametrize("new", [[3, 1], [200, 150]])
def test_cache_offsets_past_32_bits(new):
    """Blocks at both ends of a cache of 4.6 GB a side, as in a small one."""
    H, Hkv, D, bs, n = 4, 4, 128, 64, 140000
    s = step([(70, new[0]), (0, new[1])], H, Hkv, D, bs)
    small = run(s)
    check(s, small)
    blocks = s["k"][0].shape[0]
    far = torch.arange(n - blocks, n, device="cuda")
    far[:2] = torch.tensor([0, 70000])
    caches = []
    for side in "kv":
        codes, scale = torch.zeros((n, Hkv, bs, D), dtype=torch.int8, device="cuda"), torch.zeros((n, Hkv), device="cuda")
        codes[far], scale[far] = torch.from_numpy(s[side][0]).cuda(), torch.from_numpy(s[side][1]).cuda()
        caches.append((codes, scale))
    slot = torch.from_numpy(s["slot"]).cuda()
    slot = (far[slot // bs] * bs + slot % bs).to(torch.int32)
    qkv = torch.from_numpy(s["qkv"]).cuda()
    q, kc, vc = atom.atom_rotary_kv8_append(qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:], *caches, slot, *(torch.from_numpy(s[x]).cuda() for x in ("pos", "tab")))
    assert torch.equal(q, small[0])
    for got, want in ((kc, small[1]), (vc, small[2])):
        assert torch.equal(got[0][far], want[0]) and torch.equal(got[1][far], want[1])
        assert int(torch.count_nonzero(got[1])) == int(torch.count_nonzero(want[1]))


@pytest.mark.parametrize("D,bs,axes,interleaved", [(128, 64, 1, False), (64, 16, 2, True), (128, 128, 3, False), (64, 32, 1, False)])
@pytest.mark.parametrize("Hkv,n", [(3, 40), (16, 700)])
def test_single_tokens_of_many_requests(D, bs, axes, interleaved, Hkv, n):
    """Every kind of row in a batch of single tokens: zeros, large ones, scales that grow under older rows, tokens without a slot; then what is not
    finite and positions outside the table, which stay in their block and head."""
    s = step([(i * 7 % 50, 1) for i in range(n)], 2 * Hkv, Hkv, D, bs, D // 2, axes, padding=9, missing=range(3, n, 11))
    H = 2 * Hkv
    s["qkv"][5, H:] = 0
    s["qkv"][6, H:] *= 300
    s["k"][1][:] *= 0.25
    check(s, run(s, interleaved), interleaved)
    s["slot"][[2, 9]] = [s["slot"][9], s["slot"][2]]          # blocks in another order
    k = s["qkv"][:, H:H + Hkv]
    k[7, 1, 3], k[8, 0, D - 1] = np.nan, np.inf
    (s["pos"] if axes == 1 else s["pos"][0])[12] = -5
    _, kc, vc, _ = run(s, interleaved)
    with np.errstate(invalid="ignore"):
        want = ref.turned(s["qkv"][:, :H + Hkv], s["pos"], s["tab"], s["axis"], interleaved)[:, H:]
        codes, scale = kv8.append(np.where(np.isfinite(want), want, 0), *s["k"], s["slot"])
    spoilt = np.zeros(scale.shape, bool)
    for t in (7, 8, 12):
        spoilt[s["slot"][t] // bs] = ~np.isfinite(want[t]).all(1)
    assert spoilt.sum() == 2 + Hkv
    got = kc[1].cpu().numpy()
    assert np.array_equal(~np.isfinite(got), spoilt) and np.array_equal(got[~spoilt], scale[~spoilt])
    assert np.array_equal(kc[0].cpu().numpy()[~spoilt], codes[~spoilt])
    for t in (7, 8, 12):
        block, o = divmod(int(s["slot"][t]), bs)
        assert (kc[0].cpu().numpy()[block, spoilt[block], o] == 0).all()
    assert np.isfinite(vc[1].cpu().numpy()).all()
