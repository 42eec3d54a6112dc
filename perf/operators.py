"""The operators of the paged 8-bit KV cache, as measurable cases.

Three operators: the block tables and slot maps of a step built from the requests' lengths
(``map``), the step's keys and values quantised into the cache's blocks (``append``), and attention
of the step's queries over the cache (``attend``).  Each has a plain form in elementary torch
operations and, where ``own`` is true, the library's call.

A cache holds int8 codes [blocks, Hkv, block_tokens, D] and one fp32 scale for each block and head.
The definition fixes every code (IEEE fp32 steps, each rounded once), so ``append`` returns codes and
scales as they stand in the cache: whole numbers, equal on both sides, in units of their scales.
Head counts are those of the benchmark's Llama-7B, -13B and -70B shaped layers and smaller ones.
"""
import math

import torch

own = False


def listed():
    return [
        # one user's next token: a table of one row, bound by the call itself
        {"name": "map_b1", "kind": "map", "B": 1, "bs": 64, "past": 1000, "new": 1, "every": 1, "W": 64},
        # a serving step of 200 requests, every eighth a prompt of an odd length, the others decoding
        {"name": "map_b200_mixed", "kind": "map", "B": 200, "bs": 16, "past": 4000, "new": 333, "every": 8, "W": 300},
        # a large offline batch: a thousand prompts, tables wide enough for long answers
        {"name": "map_b1024_prompts", "kind": "map", "B": 1024, "bs": 32, "past": 0, "new": 256, "every": 1, "W": 1024},
        # a decoding step of 64 sequences, 32 heads
        {"name": "append_7b_b64", "kind": "append", "Hkv": 32, "D": 128, "bs": 64, "B": 64, "past": 2048, "new": 1,
         "every": 1},
        # a mixed step with small heads and blocks; rows are slices of a fused projection's output
        {"name": "append_mixed_d64", "kind": "append", "Hkv": 16, "D": 64, "bs": 16, "B": 37, "past": 900, "new": 77,
         "every": 6},
        # four prompts of up to 4096 tokens, written at once
        {"name": "append_7b_prompts", "kind": "append", "Hkv": 32, "D": 128, "bs": 64, "B": 4, "past": 0, "new": 4096,
         "every": 1},
        # one user's next token over a short context: latency
        {"name": "attend_7b_b1", "kind": "attend", "H": 32, "Hkv": 32, "D": 128, "bs": 64, "B": 1, "past": 1000,
         "new": 1, "every": 1},
        # a decoding batch, one cache head for each query head
        {"name": "attend_7b_b64", "kind": "attend", "H": 32, "Hkv": 32, "D": 128, "bs": 64, "B": 64, "past": 2048,
         "new": 1, "every": 1},
        # grouped-query heads with long contexts and short blocks
        {"name": "attend_70b_b16_long", "kind": "attend", "H": 64, "Hkv": 8, "D": 128, "bs": 16, "B": 16, "past": 16000,
         "new": 1, "every": 1},
        # a step that mixes 32 decoding requests with two chunks of prompts
        {"name": "attend_mixed", "kind": "attend", "H": 64, "Hkv": 8, "D": 128, "bs": 32, "B": 34, "past": 2000,
         "new": 500, "every": 17},
        # prompts of up to 4096 tokens, the largest compute-bound work
        {"name": "attend_70b_prompts", "kind": "attend", "H": 64, "Hkv": 8, "D": 128, "bs": 64, "B": 2, "past": 0,
         "new": 4096, "every": 1},
        # small heads: a few drafted tokens of each request checked at once, an odd count
        {"name": "attend_d64_draft", "kind": "attend", "H": 16, "Hkv": 4, "D": 64, "bs": 128, "B": 23, "past": 5000,
         "new": 5, "every": 1},
    ]


def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: the kinds in the proportion in which they are listed."""
    kind = rng.choice(["map", "append", "attend", "attend"])
    bs = rng.choice([16, 32, 64, 128])
    # decoding, prompts, or a mixture of both
    mode = rng.choice(["decode", "prompt", "mixed"])
    if kind == "map":
        B = _log(rng, 1, 1024)
        past = 0 if mode == "prompt" else _log(rng, 1, 16000)
        new = 1 if mode == "decode" else _log(rng, 2, max(2, min(4096, 200000 // B)))
        need = -(-(past + new) // bs)
        return {"kind": kind, "B": B, "bs": bs, "past": past, "new": new,
                "every": rng.randint(2, 9) if mode == "mixed" else 1, "W": min(need + _log(rng, 1, 512), max(need, (1 << 20) // B))}
    D = rng.choice([64, 128, 128])
    if kind == "append":
        Hkv = rng.choice([1, 4, 8, 16, 32, 40])
        B = _log(rng, 1, 256)
        past = 0 if mode == "prompt" else _log(rng, 1, max(1, min(8000, 6000000 // (B * Hkv))))
        new = 1 if mode == "decode" else _log(rng, 2, max(2, min(4096, 250000 // (B * Hkv))))
        return {"kind": kind, "Hkv": Hkv, "D": D, "bs": bs, "B": B, "past": past, "new": new,
                "every": rng.randint(2, 9) if mode == "mixed" else 1}
    H, Hkv = rng.choice([(32, 32), (40, 40), (64, 8), (16, 4), (20, 1), (12, 12)])
    if mode == "decode":                        # 1 to 256 sequences, up to as many keys as the largest batch has
        B = _log(rng, 1, 256)
        return {"kind": kind, "H": H, "Hkv": Hkv, "D": D, "bs": bs, "B": B,
                "past": _log(rng, 1, max(1, min(32000, 4000000 // (B * Hkv)))), "new": rng.choice([1, 1, 1, rng.randint(2, 9)]),
                "every": 1}
    if mode == "prompt":
        B = _log(rng, 1, 8)
        new = _log(rng, 20, 3000 // B)
        return {"kind": kind, "H": H, "Hkv": Hkv, "D": D, "bs": bs, "B": B, "past": rng.choice([0, _log(rng, 1, 1000)]),
                "new": new, "every": 1}
    B = _log(rng, 2, 40)
    return {"kind": kind, "H": H, "Hkv": Hkv, "D": D, "bs": bs, "B": B, "past": _log(rng, 16, 2000),
            "new": _log(rng, 2, 500), "every": rng.randint(2, 17)}


def _lengths(case):
    """(past, new) of every request: contexts spread evenly from a quarter of the longest to the
    longest; every ``every``-th request has up to ``new`` new tokens (also spread, where all have
    more than a few), the others one."""
    B, past, new, every = case["B"], case["past"], case["new"], case["every"]
    return [(_spread(past, b, B), 1 if b % every else new if new <= 16 else _spread(new, (b * 7) % B, B)) for b in range(B)]


def _spread(top, b, B):
    return top if B == 1 else top // 4 + (top - top // 4) * b // (B - 1)


def _pages(case):
    return max(-(-(p + n) // case["bs"]) for p, n in _lengths(case))


# ---- inputs -----------------------------------------------------------------------------------------


def _requests(case, g):
    """Lengths in an order of this seed; blocks in use and free ones, in a random order as in a
    cache that has served for a while; the table before the step."""
    pairs = _lengths(case)
    order = torch.randperm(len(pairs), generator=g, device="cuda")
    past, new = (torch.tensor([x[i] for x in pairs], dtype=torch.int32, device="cuda")[order].contiguous() for i in (0, 1))
    bs = case["bs"]
    W = case.get("W") or _pages(case)
    have, need = -(-past // bs), -(-(past + new) // bs)
    blocks = sum(-(-(p + n) // bs) for p, n in pairs) + 8
    ids = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    first = torch.cumsum(have, 0) - have
    j = torch.arange(W, device="cuda")[None, :]
    used = int(sum(-(-p // bs) for p, _ in pairs))
    at = (first[:, None] + j).clamp(max=blocks - 1)
    table = torch.where(j < have[:, None], ids[at], torch.full_like(ids[:1], -1)).contiguous()
    return {"past": past, "new": new, "need": need, "have": have, "table": table, "free": ids[used:].contiguous(),
            "blocks": blocks, "bs": bs, "W": W, "T": sum(n for _, n in pairs)}


def _content(r, case, g):
    """A cache whose blocks hold quantised keys and values: channels of their own mean and spread
    for the keys, as a projection with rotary positions gives them."""
    shape = (r["blocks"], case["Hkv"], r["bs"], case["D"])
    k = torch.randn(shape, generator=g, device="cuda")
    k.mul_(torch.exp(0.5 * torch.randn((1, *shape[1:2], 1, *shape[3:]), generator=g, device="cuda")))
    k.add_(torch.randn((1, *shape[1:2], 1, *shape[3:]), generator=g, device="cuda"))
    k_cache = _blocks(k)
    return k_cache, _blocks(k.normal_(generator=g).mul_(0.5))


def _blocks(x):
    s = x.abs().amax((2, 3)) / torch.full((), 127.0, device="cuda")
    return (x / s[:, :, None, None]).round_().clamp_(-127, 127).to(torch.int8), s


def _tables(r):
    """The step's table and sums, as ``map`` gives them."""
    token_start, seq_len, table, slot, _ = _map_plain(r)
    r["table"], r["token_start"], r["seq_len"], r["slot"] = table.contiguous(), token_start, seq_len, slot


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = _requests(case, g)
    r["kind"] = case["kind"]
    if case["kind"] == "map":
        return r
    _tables(r)
    r["k_cache"], r["v_cache"] = _content(r, case, g)
    T, D, Hkv = r["T"], case["D"], case["Hkv"]
    if case["kind"] == "append":                # keys and values as slices of the fused projection's output
        qkv = torch.empty((T, 3 * Hkv, D), dtype=torch.float16, device="cuda").normal_(generator=g)
        r["k"], r["v"] = qkv[:, Hkv:2 * Hkv], qkv[:, 2 * Hkv:]
        return r
    H = case["H"]
    r["q"] = torch.empty((T, H, D), dtype=torch.float16, device="cuda").normal_(generator=g)
    r["sm_scale"], r["max_new"] = D ** -0.5, max(n for _, n in _lengths(case))
    r["out"] = torch.zeros((T, H, D), dtype=torch.float16, device="cuda")
    return r


# ---- one pass ---------------------------------------------------------------------------------------


def run(state):
    if own:
        import paper_2310_19102_amd as atom
        return {"map": _map_own, "append": _append_own, "attend": _attend_own}[state["kind"]](atom, state)
    return {"map": _map_plain, "append": _append_plain, "attend": _attend_plain}[state["kind"]](state)


def _map_own(atom, s):
    token_start, seq_len, slot, cursor = atom.atom_kv_block_map(s["past"], s["new"], s["table"], s["free"], s["T"], s["bs"])
    return [token_start, seq_len, s["table"], slot, cursor]


def _append_own(atom, s):
    atom.atom_kv8_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slot"])
    return [s["k_cache"], s["v_cache"]]


def _attend_own(atom, s):
    return atom.atom_attention_kv8(s["q"], s["k_cache"], s["v_cache"], s["table"], s["token_start"], s["seq_len"],
                                   s["sm_scale"], max_new=s["max_new"], out=s["out"])


def _map_plain(s):
    past, new, bs, free, table = s["past"], s["new"], s["bs"], s["free"], s["table"]
    W, T = table.shape[1], s["T"]
    have, need = ((past + bs - 1) // bs).clamp(max=W), ((past + new + bs - 1) // bs).clamp(max=W)
    token_start = torch.zeros(past.numel() + 1, dtype=torch.int32, device=past.device)
    token_start[1:] = torch.cumsum(new, 0)
    taken = torch.cumsum(need - have, 0)
    j = torch.arange(W, device=past.device)[None, :]
    at = (taken - (need - have))[:, None] + j - have[:, None]
    fresh = torch.where(at < free.numel(), free[at.clamp(0, free.numel() - 1)], -1)
    table = torch.where(j < have[:, None], table, torch.where(j < need[:, None], fresh, -1))
    t = torch.arange(T, dtype=torch.int32, device=past.device)
    b = torch.searchsorted(token_start, t, right=True) - 1
    inside = b < past.numel()
    b = b.clamp(max=past.numel() - 1)
    p = past[b] + t - token_start[b]
    page = torch.where(inside & (p // bs < W), table[b, (p // bs).clamp(max=W - 1)], -1)
    slot = torch.where(page < 0, -1, page * bs + p % bs)
    return [token_start, (past + new).to(torch.int32), table.to(torch.int32), slot.to(torch.int32),
            taken[-1:].to(torch.int32)]


def _append_plain(s):
    bs, slot = s["bs"], s["slot"].long()
    blocks, at = torch.unique_consecutive(slot // bs, return_inverse=True)
    first = torch.full_like(blocks, bs).scatter_reduce_(0, at, slot % bs, "amin")
    return [_write_plain(s["k"].float(), *s["k_cache"], slot, bs, blocks, at, first),
            _write_plain(s["v"].float(), *s["v_cache"], slot, bs, blocks, at, first)]


def _write_plain(x, codes, scale, slot, bs, blocks, at, first):
    """Rows ``x`` into their blocks; ``first``: each block's rows before these."""
    top = torch.zeros((blocks.numel(), x.shape[1]), device=x.device).index_reduce_(0, at, x.abs().amax(2), "amax")
    old = torch.where((first > 0)[:, None], scale[blocks], 0.0)
    new = torch.maximum(old, top / torch.full_like(top, 127.0))
    r = torch.where(new > 0, 1.0 / new, 0.0)
    held = codes[blocks]
    again = (held.float() * (old / new)[:, :, None, None]).round().to(torch.int8)
    before = torch.arange(bs, device=x.device)[None, :] < first[:, None]
    keep = before[:, None, :, None] & ((new > old) & (old > 0))[:, :, None, None]
    codes[blocks] = torch.where(keep, again, held)
    codes[slot // bs, :, slot % bs] = (x * r[at][:, :, None]).round().clamp(-127, 127).to(torch.int8)
    scale[blocks] = new
    return codes, scale


def _attend_plain(s):
    q, table, token_start, seq_len, bs = s["q"], s["table"], s["token_start"], s["seq_len"], s["bs"]
    T, H, D = q.shape
    B, W = table.shape
    N, L = s["max_new"], W * bs
    pages = table.clamp(min=0).long()

    def rows(cache):                            # [B, Hkv, keys, D] in fp32
        codes, scale = cache
        x = codes[pages].float().mul_(scale[pages][..., None, None])
        return x.permute(0, 2, 1, 3, 4).reshape(B, x.shape[2], L, D)

    k = rows(s["k_cache"])
    Hkv = k.shape[1]
    i = torch.arange(N, device=q.device)
    n = token_start[1:] - token_start[:-1]
    at = (token_start[:-1, None] + i[None, :]).clamp(max=T - 1).long()
    x = q[at].float().reshape(B, N, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, (H // Hkv) * N, D)
    score = torch.matmul(x, k.transpose(2, 3)).mul_(s["sm_scale"]).view(B, Hkv, H // Hkv, N, L)
    del k, x
    last = seq_len[:, None] - n[:, None] + i[None, :]
    seen = torch.arange(L, device=q.device)[None, None, :] <= last[:, :, None]
    score.masked_fill_(~seen[:, None, None], float("-inf"))
    top = score.amax(-1, keepdim=True).clamp_(min=-1e30)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, -1, L), rows(s["v_cache"])).view(B, Hkv, H // Hkv, N, D)
    o = torch.where(total > 0, o / total, 0.0)
    t = torch.arange(T, dtype=torch.int32, device=q.device)
    b = (torch.searchsorted(token_start, t, right=True) - 1).clamp(max=B - 1)
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, N, H, D)[b, t - token_start[b]])
    return s["out"]


# ---- from the definitions, in 64 bits ---------------------------------------------------------------


def exact(case, seed):
    if case["kind"] == "map":
        return None                             # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "append":                # the scales; codes are whole numbers
        slot = s["slot"].tolist()
        got = []
        for x, (_, scale) in ((s["k"], s["k_cache"]), (s["v"], s["v_cache"])):
            x, new = x.double().abs().amax(2).cpu(), scale.double().cpu()
            seen = set()
            for t, at in enumerate(slot):
                block, row = divmod(at, s["bs"])
                if block not in seen:
                    seen.add(block)
                    if row == 0:
                        new[block] = 0.0
                new[block] = torch.maximum(new[block], x[t] / 127.0)
            got.append((None, new))
        return got
    q, bs = s["q"], s["bs"]
    T, H, D = q.shape
    out = torch.zeros((T, H, D), dtype=torch.float64, device="cuda")
    start, length, table = s["token_start"].tolist(), s["seq_len"].tolist(), s["table"].tolist()
    group = H // case["Hkv"]
    for b in range(case["B"]):
        L, n = length[b], start[b + 1] - start[b]
        pages = torch.tensor(table[b][:-(-L // bs)], device="cuda")
        seen = torch.arange(L, device="cuda")[None, :] <= (L - n + torch.arange(n, device="cuda"))[:, None]
        for h in range(case["Hkv"]):
            k, v = ((c[pages, h].double() * sc[pages, h].double()[:, None, None]).reshape(-1, D)[:L]
                    for c, sc in (s["k_cache"], s["v_cache"]))
            for j in range(h * group, (h + 1) * group):
                e = (q[start[b]:start[b + 1], j].double() @ k.T.contiguous()) * s["sm_scale"]
                w = torch.softmax(e.masked_fill(~seen, float("-inf")), -1)
                out[start[b]:start[b + 1], j] = w @ v
    return out


# ---- what a pass cannot do without ------------------------------------------------------------------


def work(case):
    """Inputs read once, outputs written once; two operations per multiply-add."""
    pairs = _lengths(case)
    bs, T = case["bs"], sum(n for _, n in pairs)
    have, need, full = (sum(x) for x in zip(*((-(-p // bs), -(-(p + n) // bs), p // bs) for p, n in pairs)))
    B = len(pairs)
    if case["kind"] == "map":
        return {"bytes": 8 * B + 4 * (need - have) + 4 * (B * case["W"] - have) + 8 * B + 4 * T, "flops": 0}
    Hkv, D = case["Hkv"], case["D"]
    if case["kind"] == "append":
        scales = 8 * Hkv * ((need - full) + (have - full))      # written, and read where a block has older rows
        return {"bytes": T * (6 * Hkv * D + 4) + scales, "flops": 4 * T * Hkv * D}
    H = case["H"]
    keys = sum(p + n for p, n in pairs)
    seen = sum(n * p + n * (n + 1) // 2 for p, n in pairs)
    return {"bytes": keys * 2 * Hkv * D + need * (8 * Hkv + 4) + 4 * T * H * D + 8 * B, "flops": 4 * seen * H * D}
