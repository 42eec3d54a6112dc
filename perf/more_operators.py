"""The operators of a decoding layer whose activations stay in fp16, as measurable cases.

Four operators: rotary positions of one or several axes (``rotary``), the same fused with the append to the paged 8-bit
cache (``append``), linear layers with the 4-bit weights of this library and fp16 activations (``linear``), and the gated
half of the feed-forward block on such weights (``gated``).  Each has a plain form in elementary torch operations and, where
``own`` is true, the library's call.

``append`` defines every code of the cache (IEEE fp32 steps, each rounded once), so it returns them as they stand there:
whole numbers, equal on both sides, in units of the scales beside them.  Head counts, layer sizes and heavy-tailed
activations are those of the benchmark's Llama-7B, -13B and -70B shaped layers, and smaller ones.
"""
import math

import torch

own = False


def listed():
    return [
        # one user's next token, 32 query and 32 key heads of the fused projection: bound by the call itself
        {"name": "rotary_7b_b1", "kind": "rotary", "T": 1, "heads": 64, "D": 128, "R": 128, "axes": 1, "interleaved": False,
         "transposed": False, "P": 4096},
        # frames of a video: time, height and width, 64 query heads on 8 key heads
        {"name": "rotary_video", "kind": "rotary", "T": 4999, "heads": 72, "D": 128, "R": 128, "axes": 3, "interleaved": False,
         "transposed": False, "P": 8192},
        # the gradient's way through positions that turn half of small heads, neighbouring channels a pair
        {"name": "rotary_d64_back", "kind": "rotary", "T": 3001, "heads": 20, "D": 64, "R": 32, "axes": 1, "interleaved": True,
         "transposed": True, "P": 16384},
        # a decoding step of 64 sequences, 32 heads
        {"name": "append_7b_b64", "kind": "append", "H": 32, "Hkv": 32, "D": 128, "R": 128, "axes": 1, "interleaved": False, "bs": 64,
         "B": 64, "past": 2048, "new": 1, "every": 1},
        # a step that mixes 37 requests, every sixth a chunk with image tokens, grouped heads and short blocks
        {"name": "append_mixed_axes", "kind": "append", "H": 64, "Hkv": 8, "D": 128, "R": 128, "axes": 3, "interleaved": False, "bs": 16,
         "B": 37, "past": 900, "new": 277, "every": 6},
        # four prompts of up to 4096 tokens, turned and written at once
        {"name": "append_7b_prompts", "kind": "append", "H": 32, "Hkv": 32, "D": 128, "R": 128, "axes": 1, "interleaved": False, "bs": 64,
         "B": 4, "past": 0, "new": 4096, "every": 1},
        # one user's next token through an attention output projection, with the residual
        {"name": "linear_7b_m1", "kind": "linear", "M": 1, "K": 4096, "N": 4096, "norm": False, "index": True, "residual": True},
        # eight sequences through the fused QKV projection behind the norm
        {"name": "linear_7b_qkv_m8", "kind": "linear", "M": 8, "K": 4096, "N": 12288, "norm": True, "index": True, "residual": False},
        # a batch through a long down projection whose input comes in reordered order
        {"name": "linear_70b_down_m33", "kind": "linear", "M": 33, "K": 28672, "N": 8192, "norm": False, "index": False, "residual": True},
        # one user's next token through the gated half of the feed-forward block
        {"name": "gated_7b_m1", "kind": "gated", "M": 1, "K": 4096, "N": 11008, "norm": True, "index": True},
        # an odd batch and an odd number of channels, as one of several GPUs holds them
        {"name": "gated_13b_part_m5", "kind": "gated", "M": 5, "K": 5120, "N": 3455, "norm": True, "index": True},
        # the largest batch
        {"name": "gated_70b_m64", "kind": "gated", "M": 64, "K": 8192, "N": 28672, "norm": True, "index": True},
    ]


def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: the kinds in the proportion in which they are listed."""
    kind = rng.choice(["rotary", "append", "linear", "gated"])
    if kind in ("linear", "gated"):
        M = _log(rng, 1, 64)
        K = 128 * _log(rng, 4, 224 if kind == "linear" else 64)
        N = _log(rng, 64, min(28672, 28672 * 8192 // K))
        case = {"kind": kind, "M": M, "K": K, "N": N, "norm": rng.random() < 0.5, "index": rng.random() < 0.75}
        return {**case, "residual": rng.random() < 0.5} if kind == "linear" else case
    D = rng.choice([64, 128, 128])
    R = rng.choice([D, D, D // 2, D // 4])
    turn = {"D": D, "R": R, "axes": rng.choice([1, 1, 2, 3, 4]), "interleaved": rng.random() < 0.3}
    if kind == "rotary":
        heads = rng.choice([1, 5, 8, 20, 40, 64, 72])
        return {"kind": kind, "T": _log(rng, 1, min(8192, 5000 * 72 // heads)), "heads": heads, **turn, "transposed": rng.random() < 0.3,
                "P": _log(rng, 512, 32768)}
    bs = rng.choice([16, 32, 64, 128])
    H, Hkv = rng.choice([(32, 32), (40, 40), (64, 8), (16, 4), (20, 1), (12, 12)])
    mode = rng.choice(["decode", "prompt", "mixed"])        # decoding, prompts, or a mixture of both
    B = _log(rng, 1, 256)
    past = 0 if mode == "prompt" else _log(rng, 1, max(1, min(8000, 6000000 // (B * Hkv))))
    new = 1 if mode == "decode" else _log(rng, 2, max(2, min(4096, 250000 // (B * max(Hkv, H // 2)))))
    return {"kind": kind, "H": H, "Hkv": Hkv, **turn, "bs": bs, "B": B, "past": past, "new": new,
            "every": rng.randint(2, 9) if mode == "mixed" else 1}


def _lengths(case):
    """(past, new) of every request: contexts spread evenly from a quarter of the longest to the longest; every ``every``-th
    request has up to ``new`` new tokens (also spread, where they have more than a few), the others one."""
    B, past, new, every = case["B"], case["past"], case["new"], case["every"]
    return [(_spread(past, b, B), 1 if b % every else new if new <= 16 else _spread(new, (b * 7) % B, B)) for b in range(B)]


def _spread(top, b, B):
    return top if B == 1 else top // 4 + (top - top // 4) * b // (B - 1)


# ---- inputs -----------------------------------------------------------------------------------------


def _axes(case):
    """Each pair's axis: the pairs shared out among the axes in turn, the first axis a little fewer."""
    n, A = case["R"] // 2, case["axes"]
    return tuple(min(A - 1, j * A // n if A < 3 else (0 if 4 * j < n else 1 + (4 * j - n) * (A - 1) // (3 * n))) for j in range(n))


def _coordinates(p, A):
    """The axes' positions of tokens at p: text counts on all axes alike; where there are several, runs of 576 image tokens
    have a frame's number, a row and a column instead."""
    if A == 1:
        return p[None].contiguous()
    image = (p // 576) % 2 == 1
    base, at = p // 576 * 576, p % 576
    rows = [torch.where(image, base, p), torch.where(image, base + at // 24, p), torch.where(image, base + at % 24, p), p]
    return torch.stack(rows[:A]).to(torch.int32).contiguous()


def _table(case, P):
    """cos and sin of position times frequency, [P, R / 2, 2]; the angles in 64 bits."""
    n = case["R"] // 2
    f = 10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)
    angle = torch.arange(P, dtype=torch.float64, device="cuda")[:, None] * f[None, :]
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


def _turning(case, p, P):
    return {"positions": _coordinates(p, case["axes"]), "table": _table(case, P), "axis": bytes(_axes(case)),
            "axis_of": torch.tensor(_axes(case), device="cuda"), "R": case["R"], "interleaved": case["interleaved"]}


def _prepare_rotary(case, g):
    T, heads, D, P = case["T"], case["heads"], case["D"], case["P"]
    x = torch.empty((T, heads + heads // 4 + 1, D), dtype=torch.float16, device="cuda").normal_(generator=g)
    first = int(torch.randint(0, max(1, P - T), (1,), generator=g, device="cuda"))
    p = ((first + torch.arange(T, device="cuda")) % P).to(torch.int32)
    return {**_turning(case, p, P), "x": x[:, :heads], "transposed": case["transposed"],
            "out": torch.zeros((T, heads, D), dtype=torch.float16, device="cuda")}


def _prepare_append(case, g):
    """Queries, keys and values as slices of the fused projection's output; blocks in a random order as in a cache that has
    served for a while, older rows in them."""
    pairs = _lengths(case)
    H, Hkv, D, bs = case["H"], case["Hkv"], case["D"], case["bs"]
    order = torch.randperm(len(pairs), generator=g, device="cuda").tolist()
    pairs = [pairs[i] for i in order]
    T = sum(n for _, n in pairs)
    need = [-(-(p + n) // bs) for p, n in pairs]
    blocks = sum(need) + 8
    ids = torch.randperm(blocks, generator=g, device="cuda")
    past = torch.tensor([p for p, _ in pairs], device="cuda")
    new = torch.tensor([n for _, n in pairs], device="cuda")
    first = torch.cumsum(torch.tensor(need, device="cuda"), 0) - torch.tensor(need, device="cuda")
    b = torch.repeat_interleave(torch.arange(len(pairs), device="cuda"), new)
    p = past[b] + torch.arange(T, device="cuda") - (torch.cumsum(new, 0) - new)[b]
    slot = (ids[first[b] + p // bs] * bs + p % bs).to(torch.int32)
    qkv = torch.empty((T, H + 2 * Hkv, D), dtype=torch.float16, device="cuda").normal_(generator=g)
    caches = []
    for spread in (1.0, 0.5):
        codes = torch.randint(-127, 128, (blocks, Hkv, bs, D), generator=g, device="cuda", dtype=torch.int8)
        caches.append((codes, torch.rand((blocks, Hkv), generator=g, device="cuda").add_(3.0).mul_(spread / 127)))
    P = max(p + n for p, n in pairs)
    return {**_turning(case, p.to(torch.int32), P), "q": qkv[:, :H], "k": qkv[:, H:H + Hkv], "v": qkv[:, H + Hkv:], "slot": slot.contiguous(),
            "k_cache": caches[0], "v_cache": caches[1], "bs": bs, "out": torch.zeros((T, H, D), dtype=torch.float16, device="cuda")}


def _weights(N, K, g):
    """Codes and scales of N rows as the quantisation of weights gives them: 128 outlier channels in 8 bits, the others in
    4, two in a byte, a scale for each 128."""
    G, K4 = K // 128, K - 128
    scale = torch.empty((N, G), device="cuda").normal_(generator=g).mul_(0.1).add_(1.0).mul_(0.006)
    scale[:, -1] *= 1.0 / 16
    q8 = torch.empty((N, 128), device="cuda").normal_(generator=g).mul_(45).round_().clamp_(-128, 127).to(torch.int8)
    q4 = torch.empty((N, K4), dtype=torch.float16, device="cuda").normal_(generator=g).mul_(2.8).round_().clamp_(-8, 7).to(torch.int8)
    q4 = ((q4[:, 1::2] << 4) | (q4[:, 0::2] & 15)).view(torch.uint8)
    return q4.contiguous(), q8, scale.half()


def _prepare_product(case, g):
    """Activations with channels of very different sizes, the largest last in the order of the index."""
    M, K, N = case["M"], case["K"], case["N"]
    size = torch.exp(torch.empty(K, device="cuda").normal_(generator=g))
    order = torch.argsort(size).to(torch.int32)
    if not case["index"]:
        size = size[order.long()]
    x = torch.empty((M, K), device="cuda").normal_(generator=g).mul_(size).half()
    s = {"x": x, "gamma": None, "index": order if case["index"] else None, "residual": None, "eps": 1e-6,
         "weights": [_weights(N, K, g) for _ in range(2 if case["kind"] == "gated" else 1)],
         "out": torch.zeros((M, N), dtype=torch.float16, device="cuda")}
    if case["norm"]:
        s["gamma"] = torch.empty(K, device="cuda").normal_(generator=g).mul_(0.1).add_(1.0).half()
    if case.get("residual"):
        s["residual"] = torch.empty((M, N), dtype=torch.float16, device="cuda").normal_(generator=g)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = {"rotary": _prepare_rotary, "append": _prepare_append}.get(case["kind"], _prepare_product)
    return {"kind": case["kind"], **make(case, g)}


# ---- one pass ---------------------------------------------------------------------------------------


def run(state):
    if own:
        import paper_2310_19102_amd as atom
        return {"rotary": _rotary_own, "append": _append_own, "linear": _linear_own, "gated": _gated_own}[state["kind"]](atom, state)
    return {"rotary": _rotary_plain, "append": _append_plain, "linear": _linear_plain, "gated": _gated_plain}[state["kind"]](state)


def _rotary_own(atom, s):
    return atom.atom_rotary(s["x"], s["positions"], s["table"], axis=s["axis"], interleaved=s["interleaved"],
                            transposed=s["transposed"], out=s["out"])


def _append_own(atom, s):
    q, k_cache, v_cache = atom.atom_rotary_kv8_append(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["slot"], s["positions"],
                                                      s["table"], axis=s["axis"], interleaved=s["interleaved"], out=s["out"])
    return [q, k_cache, v_cache]


def _linear_own(atom, s):
    return atom.atom_w4a16_linear(s["x"], s["gamma"], s["eps"], s["index"], *s["weights"][0], residual=s["residual"], out=s["out"])


def _gated_own(atom, s):
    return atom.atom_w4a16_swiglu(s["x"], s["gamma"], s["eps"], s["index"], *s["weights"], out=s["out"])


def _turned(s, x, transposed=False):
    """x [T, heads, D] in fp32, turned; every product and sum rounded once."""
    n = s["R"] // 2
    at = s["positions"].long()[s["axis_of"]]                                 # [pairs, T]
    c, d = s["table"][at.T, torch.arange(n, device=x.device)[None, :]].unbind(-1)
    c, d = c[:, None], (-d if transposed else d)[:, None]
    turn, rest = x[..., :2 * n].float(), x[..., 2 * n:].float()
    a, b = (turn[..., 0::2], turn[..., 1::2]) if s["interleaved"] else (turn[..., :n], turn[..., n:])
    u, w = a * c - b * d, b * c + a * d
    return torch.cat([torch.stack([u, w], -1).flatten(-2) if s["interleaved"] else torch.cat([u, w], -1), rest], -1)


def _rotary_plain(s):
    return s["out"].copy_(_turned(s, s["x"], s["transposed"]))


def _append_plain(s):
    bs, slot = s["bs"], s["slot"].long()
    blocks, at = torch.unique_consecutive(slot // bs, return_inverse=True)
    first = torch.full_like(blocks, bs).scatter_reduce_(0, at, slot % bs, "amin")
    return [s["out"].copy_(_turned(s, s["q"])), _written(_turned(s, s["k"]), *s["k_cache"], slot, bs, blocks, at, first),
            _written(s["v"].float(), *s["v_cache"], slot, bs, blocks, at, first)]


def _written(x, codes, scale, slot, bs, blocks, at, first):
    """Rows x into their blocks; ``first``: each block's rows before these."""
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


def _activations(s):
    x = s["x"].float()
    if s["gamma"] is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * s["gamma"].float()
    return x if s["index"] is None else x[:, s["index"].long()]


def _product(x, weights):
    q4, q8, scale = weights
    code = torch.stack([(q4 & 15).view(torch.int8), (q4 >> 4).view(torch.int8)], -1).flatten(1)
    code = torch.cat([torch.where(code > 7, code - 16, code), q8], 1).float()
    w = code.view(code.shape[0], -1, 128).mul_(scale.float()[:, :, None]).view(code.shape)
    return x @ w.T


def _linear_plain(s):
    y = _product(_activations(s), s["weights"][0])
    return s["out"].copy_(y if s["residual"] is None else y + s["residual"].float())


def _gated_plain(s):
    x = _activations(s)
    gate, up = (_product(x, w) for w in s["weights"])
    return s["out"].copy_(gate / (1.0 + torch.exp(-gate)) * up)


# ---- from the definitions, in 64 bits ---------------------------------------------------------------


def _turned_exactly(case, s, x, transposed=False):
    """Each pair as a complex number, turned by its own angle."""
    n = case["R"] // 2
    f = 10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)
    pos = torch.stack([s["positions"][a] for a in _axes(case)], 1).double()  # [T, pairs]
    turn = torch.polar(torch.ones_like(pos), (-1.0 if transposed else 1.0) * pos * f)[:, None]
    y = x.double().clone()
    lo, hi = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if case["interleaved"] else (slice(0, n), slice(n, 2 * n))
    z = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * turn
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def _product_exactly(x, weights, rows=2048):
    """A group at a time: its codes' sum of products, times its scale."""
    q4, q8, scale = weights
    y = torch.empty((x.shape[0], q8.shape[0]), dtype=torch.float64, device="cuda")
    for n in range(0, q8.shape[0], rows):
        low, high = q4[n:n + rows].int() % 16, q4[n:n + rows].int() // 16
        codes = torch.empty((low.shape[0], x.shape[1]), dtype=torch.float64, device="cuda")
        codes[:, 0:2 * low.shape[1]:2] = low - 16 * (low // 8)
        codes[:, 1:2 * low.shape[1]:2] = high - 16 * (high // 8)
        codes[:, 2 * low.shape[1]:] = q8[n:n + rows]
        y[:, n:n + rows] = sum((x[:, 128 * j:128 * j + 128] @ codes[:, 128 * j:128 * j + 128].T) * scale[n:n + rows, j].double()
                               for j in range(scale.shape[1]))
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return _turned_exactly(case, s, s["x"], case["transposed"])
    if case["kind"] == "append":                # the queries and the scales; codes are whole numbers
        got = [_turned_exactly(case, s, s["q"])]
        slot = s["slot"].tolist()
        for x, (_, scale) in ((_turned_exactly(case, s, s["k"]), s["k_cache"]), (s["v"].double(), s["v_cache"])):
            x, new, seen = x.abs().amax(2).cpu(), scale.double().cpu(), set()
            for t, at in enumerate(slot):
                block, row = divmod(at, s["bs"])
                if block not in seen:
                    seen.add(block)
                    if row == 0:
                        new[block] = 0.0
                new[block] = torch.maximum(new[block], x[t] / 127.0)
            got.append((None, new))
        return got
    x = s["x"].double()
    if s["gamma"] is not None:
        x = x / torch.sqrt(x.square().mean(1, keepdim=True) + s["eps"]) * s["gamma"].double()
    if s["index"] is not None:
        x = torch.index_select(x, 1, s["index"])
    y = [_product_exactly(x, w) for w in s["weights"]]
    if case["kind"] == "gated":
        return y[0] * torch.sigmoid(y[0]) * y[1]
    return y[0] if s["residual"] is None else y[0] + s["residual"].double()


# ---- what a pass cannot do without ------------------------------------------------------------------


def work(case):
    """Inputs read once, outputs written once; two operations per multiply-add, six for a pair that turns."""
    if case["kind"] in ("linear", "gated"):
        M, K, N = case["M"], case["K"], case["N"]
        n = 2 if case["kind"] == "gated" else 1
        small = 2 * K * case["norm"] + 4 * K * case["index"] + 2 * M * N * bool(case.get("residual"))
        return {"bytes": n * N * ((K - 128) // 2 + 128 + K // 64) + 2 * M * K + 2 * M * N + small, "flops": 2 * n * M * K * N}
    if case["kind"] == "rotary":
        T, rows, out = case["T"], case["T"] * case["heads"] * case["D"], 4
        turned, used, scales = case["T"] * case["heads"], min(case["T"], case["P"]), 0
    else:
        pairs, bs = _lengths(case), case["bs"]
        T = sum(n for _, n in pairs)
        touched = sum(-(-(p + n) // bs) - p // bs for p, n in pairs)
        H, Hkv, D = case["H"], case["Hkv"], case["D"]
        rows, out, turned, scales = T * D, 4 * H + 6 * Hkv, T * (H + Hkv), 8 * Hkv * touched + 4 * T
        used = min(T, max(p + n for p, n in pairs))
    return {"bytes": rows * out + used * 4 * case["R"] + 4 * case["axes"] * T + scales, "flops": 3 * case["R"] * turned}
