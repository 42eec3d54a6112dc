"""Attention over the paged 8-bit cache with contexts of many keys, where the general bound on rounding has become wider than a key: caches whose
outputs say which keys were read, and how often."""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import Case, i32, npy

pytestmark = pytest.mark.gpu

# (H, Hkv, D, bs, past, new, extra columns)
LONG = [
    (8, 1, 64, 32, [20000], [1], 1), (64, 8, 128, 16, [5000, 17], [1, 1], 1), (4, 4, 128, 128, [4000, 3], [2, 9], 1), (16, 4, 64, 16, [3000], [64], 1),
    (16, 16, 128, 32, [10, 2000, 0], [1, 200, 90], 1), (64, 8, 128, 64, [0], [300], 1), (20, 1, 64, 32, [2000, 3000], [2, 3], 3000),
    (4, 1, 128, 128, [5000, 2999, 40], [1, 30, 16], 3000), (2, 2, 128, 16, [9000], [100], 3000), (8, 8, 64, 32, [4500, 100, 4200], [1, 200, 2], 3000),
    (128, 1, 128, 32, [6500], [100], 1), (128, 1, 64, 32, [1300], [500], 1), (64, 8, 128, 64, [1100], [1500], 1), (3, 3, 128, 128, [5000, 2, 0], [11, 21, 32], 2048),
    (16, 4, 64, 128, [5000, 4000, 2500], [5, 5, 5], 1), (32, 32, 128, 64, [1000], [1], 1), (2, 1, 128, 64, [37777], [1], 9)]


def positions(c, b):
    """The blocks and rows of the request's keys, in their order."""
    bs = c.kc[0].shape[2]
    p = torch.arange(int(c.len[b]), device="cuda")
    return c.table[b, p // bs].long(), p % bs


@pytest.mark.parametrize("H,Hkv,D,bs,past,new,extra", LONG)
def test_every_visible_key_counts_once(H, Hkv, D, bs, past, new, extra):
    """Queries of zeros: every weight is the same power of two, so sums are exact, and the output is the mean of the visible values.  Key s has 127 in dimension
    s % D and 0 elsewhere: a dimension's mean tells how many of its keys were added.  Off are the output's rounding (2^-11) and three of the quotient (2^-22
    of it together); a key more or less is 1 / (keys / D), 2^-9 at 37777 keys, or more."""
    c = Case(H, Hkv, D, bs, past, new, seed=1, extra=extra)
    c.q.zero_()
    c.vc[1].fill_(2.0 ** -7)
    c.vc[0].fill_(-99)                                      # rows behind a request's last
    for b, (p, n) in enumerate(zip(past, new)):
        pages, rows = positions(c, b)
        s = torch.arange(p + n, device="cuda")
        c.vc[0][pages, :, rows] = torch.nn.functional.one_hot(s % D, D).to(torch.int8)[:, None, :] * 127
    got = npy(c.call()).astype(np.float64)
    at = 0
    for p, n in zip(past, new):
        seen = p + 1 + np.arange(n)                         # of each query
        count = (seen[:, None] - np.arange(D)[None, :] + D - 1) // D
        want = (127 * 2.0 ** -7 * count / seen[:, None])[:, None, :]
        off = np.abs(got[at:at + n] - want)
        assert (off <= (2.0 ** -11 + 2.0 ** -21) * want).all(), f"{(off / np.maximum(want, 1e-9)).max():.2e}"
        at += n


@pytest.mark.parametrize("H,Hkv,D,bs,past,new,extra", LONG)
def test_a_query_finds_its_key(H, Hkv, D, bs, past, new, extra):
    """Keys of random signs, each query one of them times a factor that makes its weight 2^30 of all others' together, or more: the output is that key's value.  Keys on both
    sides of every multiple of 128 (where pieces are cut) in turn, the first and the last that a query sees.  Off are the weight's rounding and the output's, 2^-11
    each, and the others' weights."""
    c = Case(H, Hkv, D, bs, past, new, seed=2, extra=extra)
    g = torch.Generator().manual_seed(H + D)
    group = H // Hkv
    c.kc[0].copy_(torch.randint(0, 2, c.kc[0].shape, generator=g) * 254 - 127)
    c.kc[1].fill_(1.0 / 128)
    c.sm = 1.0
    targets = torch.zeros((c.T, H), dtype=torch.long)
    at, heads, want = 0, torch.arange(H) // group, torch.zeros((c.T, H, D), dtype=torch.float64)
    for b, (p, n) in enumerate(zip(past, new)):
        pages, rows = positions(c, b)
        k, v = (cache[0][pages, :, rows].cpu() for cache in (c.kc, c.vc))      # [keys, Hkv, D]
        vs = c.vc[1][pages].cpu()
        for i in range(n):
            last = p + i
            edges = [s for m in range(128, last + 2, 128) for s in (m - 1, m) if s <= last]
            pick = [0, last, *edges, *torch.randint(0, last + 1, (8,), generator=g).tolist()]
            s = torch.tensor([pick[(i * H + h) % len(pick)] for h in range(H)])
            targets[at + i] = s
            c.q[at + i] = (4.0 * torch.sign(k[s, heads].float())).to(torch.float16).cuda()
            want[at + i] = v[s, heads].double() * vs[s, heads].double()[:, None]
        # the gap, of this request's last query: binary orders between its key and the sum of the others
        e = (c.q[at + n - 1].double().view(Hkv, group, D).cpu() @ k.double().permute(1, 2, 0).contiguous()).view(H, -1) / 128 * np.log2(np.e)
        top = e.gather(1, targets[at + n - 1][:, None])
        rest = torch.exp2(e - top).sum(1) - 1
        assert (rest < 2.0 ** -30).all()
        at += n
    got = c.call().double().cpu()
    off = (got - want).abs()
    assert (off <= (2 * 2.0 ** -11 + 2.0 ** -20) * want.abs() + 2.0 ** -25).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hkv,past,new,few", [(8, 8, 1 << 16, [1] * 140, True), (64, 8, 65000, [1100], False)])
def test_many_small_weights_beside_a_large_one(H, Hkv, past, new, few, D):
    """A first key that every query attends to and whose value is zero, and 65000 others with weights of 2^-22.68 of its: the output is what these add up to, 1 % of their
    value.  A weight travels as fp16, off by 2^-11 of itself or 2^-30 of the largest; here 2^-30 / 2^-22.68 = 0.6 %, the same for all of them.  The output's own
    rounding is 2^-11, of the exponents 24 * 2^-23 at most, the sums' 2^-12 of a chain of 2048 additions."""
    bs, keys = 128, past + max(new)
    c = Case(H, Hkv, D, bs, [bs], [0], seed=1)              # two blocks: the first keys, and one that stands for all others
    q0 = 15.71875
    B, T = len(new), sum(new)
    table = torch.ones((B, -(-keys // bs)), dtype=torch.int32, device="cuda")
    table[:, 0] = 0
    c.kc[0].zero_()
    c.kc[0][0, :, 0, 0] = 64                                # its score is q0, theirs 0
    c.kc[1].fill_(2.0 ** -6)
    c.vc[0].fill_(100)
    c.vc[0][0, :, 0] = 0
    c.vc[1].fill_(2.0 ** -6)
    c.q = torch.zeros((T, H, D), dtype=torch.float16, device="cuda")
    c.q[:, :, 0] = q0
    c.table, c.T, c.max_new, c.sm, c.W = table, T, max(new), 1.0, table.shape[1]
    c.start = i32(*np.concatenate([[0], np.cumsum(new)]).tolist())
    c.len = i32(*[past + n for n in new])
    assert c.route()[1:] == (False, not few, False)
    got = npy(c.call()).astype(np.float64)
    seen = np.concatenate([past + 1 + np.arange(n) for n in new])
    others = (seen - 1) * np.exp(-q0)
    want = (others / (1 + others) * 100 * 2.0 ** -6)[:, None, None]
    rel = 2.0 ** -11 + 2.0 ** -30 * np.exp(q0) + 2.0 ** -11 + 24 * 2.0 ** -23 + 2.0 ** -12
    assert (np.abs(got - want) <= rel * want).all(), np.abs(got / want - 1).max()
