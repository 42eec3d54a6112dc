"""The paged 8-bit KV cache in plain numpy: tables and codes by the definition (IEEE fp32 steps), attention in 64 bits with
the error that its fp16 weights and output may have."""
import numpy as np


def block_map(past, new, table, free, T, bs, cursor=0):
    """(token_start, seq_len, slot, cursor_out, table) of one step."""
    B, W = table.shape
    table = table.copy()
    past, new = [max(0, int(p)) for p in past], [max(0, int(n)) for n in new]
    start, slot, f, total = [0], np.full(T, -1, np.int64), int(cursor), 0
    for b in range(B):
        have, need = min(W, -(-past[b] // bs)), min(W, -(-(past[b] + new[b]) // bs))
        for j in range(have, W):
            table[b, j] = -1
            if j < need:
                table[b, j] = free[f] if 0 <= f < len(free) else -1
                f += 1
        for i in range(new[b]):
            t, p = total + i, past[b] + i
            if t < T and p // bs < W and table[b, p // bs] >= 0:
                slot[t] = int(table[b, p // bs]) * bs + p % bs
        total += new[b]
        start.append(total)
    return (np.array(start, np.int32), np.array([p + n for p, n in zip(past, new)], np.int32), slot.astype(np.int32),
            np.array([f], np.int32), table)


def append(x, codes, scale, slot):
    """One of the two caches after the rows x [T, Hkv, D] fp16; codes [n, Hkv, bs, D], scale [n, Hkv]."""
    codes, scale = codes.copy(), scale.copy()
    n, _, bs, _ = codes.shape
    x = x.astype(np.float32)
    inside = lambda s: 0 <= s < n * bs                      # noqa: E731
    t = 0
    while t < len(slot):
        if not inside(slot[t]):
            t += 1
            continue
        block, o = divmod(int(slot[t]), bs)
        end = t + 1
        while end < len(slot) and slot[end] == slot[end - 1] + 1 and slot[end] % bs:
            end += 1
        run = x[t:end]                                      # [len, Hkv, D]
        s_old = scale[block] if o else np.zeros_like(scale[block])
        s = np.maximum(s_old, np.abs(run).max((0, 2)) / np.float32(127))
        with np.errstate(divide="ignore", invalid="ignore"):
            r = np.where(s > 0, np.float32(1) / s, np.float32(0)).astype(np.float32)
            ratio = (s_old / s).astype(np.float32)
        for h in np.nonzero((s > s_old) & (s_old > 0))[0]:
            codes[block, h, :o] = np.rint(codes[block, h, :o].astype(np.float32) * ratio[h]).astype(np.int8)
        codes[block, :, o:o + end - t] = np.clip(np.rint(run * r[None, :, None]), -127, 127).astype(np.int8).transpose(1, 0, 2)
        scale[block] = s
        t = end
    return codes, scale


def attention(q, k_cache, v_cache, table, token_start, seq_len, sm_scale, max_new=None):
    """(out [T, H, D] in 64 bits, bound on the error of each element, rows that are computed)."""
    T, H, D = q.shape
    (kc, ks), (vc, vs) = k_cache, v_cache
    n_blocks, Hkv, bs, _ = kc.shape
    B, W = table.shape
    g = H // Hkv
    q = q.astype(np.float64)
    out, tol, done = np.zeros((T, H, D)), np.zeros((T, H, D)), np.zeros(T, bool)
    for b in range(B):
        first, end = int(token_start[b]), int(token_start[b + 1])
        n, L = end - first, int(seq_len[b])
        keys = min(max(L, 0), W * bs)
        pages = table[b, :-(-keys // bs)]
        there = np.repeat((pages >= 0) & (pages < n_blocks), bs)[:keys]
        at = np.where((pages >= 0) & (pages < n_blocks), pages, 0)
        computed = [i for i in range(n) if first + i < T and (max_new is None or i < max_new)]
        if not computed:
            continue
        done[first + computed[0]:first + computed[-1] + 1] = True
        for h in range(Hkv):
            kh = (kc[at, h].astype(np.float64) * np.nan_to_num(ks[at, h]).astype(np.float64)[:, None, None]).reshape(-1, D)[:keys]
            vh = (vc[at, h].astype(np.float64) * np.nan_to_num(vs[at, h]).astype(np.float64)[:, None, None]).reshape(-1, D)[:keys]
            vmax = 127 * np.repeat(np.nan_to_num(vs[at, h]).astype(np.float64), bs)[:keys]
            kmax = np.where(there, np.repeat(np.nan_to_num(ks[at, h]).astype(np.float64), bs)[:keys], 0)
            for i in computed:
                see = there & (np.arange(keys) <= L - n + i)
                if not see.any():
                    continue
                for j in range(h * g, (h + 1) * g):
                    x = q[first + i, j]
                    e = (kh[see] @ x) * sm_scale
                    top = e.max()
                    w = np.exp(e - top)
                    w /= w.sum()
                    o = w @ vh[see]
                    out[first + i, j] = o
                    # sum of |weight * value|: what relative errors of the weights and sums act on
                    mass = w @ np.abs(vh[see])
                    # scores: D products of q with codes + 128 (255 at most) and the offset, added in fp32
                    score = sm_scale * kmax[see].max() * 256 * np.abs(x).sum() * (D + 2) * 2.0 ** -24
                    # exponent: its argument is rounded a few times, 2^x and log2 are good to an ulp
                    arg = 8 * 2.0 ** -24 * (np.abs(e).max() * 1.5 + 60)
                    sums = 2.0 ** -24 * (keys + 64)         # fp32 sums of the weights and of the products
                    rel = 2.0 ** -11 + 2 * (score + arg) + 2 * sums
                    tiny = 2.0 ** -25 * (w * vmax[see]).max() * 127 / 127 * keys   # weights below fp16's normal numbers
                    tol[first + i, j] = 2.0 ** -11 * np.abs(o) + rel * mass + tiny + 2.0 ** -25
    return out, tol, done
