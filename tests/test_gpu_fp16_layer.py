"""A decoding layer whose activations stay fp16, as its calls are used together: two linear layers on 4-bit weights around the
rotary append and the attention, two more around the gated product; prompts, mixed steps and single tokens."""
import ctypes

import numpy as np
import pytest
import torch

import _fp16_layer_ref as ref
import _kv8_ref as kv8
import paper_2310_19102_amd as atom

pytestmark = pytest.mark.gpu

EPS, H, HKV, D, FFN, BS, W, PAIRS, P = 1e-5, 8, 2, 64, 640, 16, 12, 24, 256
HIDDEN = H * D


def npy(t):
    return t.detach().cpu().numpy()


def weights(N, K, rng):
    """About the size of a trained layer's: results keep the size of what goes in."""
    scale = (0.2 / np.sqrt(K) * (1 + 0.2 * rng.random((N, K // 128)))).astype(np.float16)
    q4, q8 = rng.integers(0, 256, (N, (K - 128) // 2)).astype(np.uint8), rng.integers(-20, 21, (N, 128)).astype(np.int8)
    return tuple(torch.from_numpy(a).cuda() for a in (q4, q8, scale))


class Server:
    """One layer, its cache, and up to B requests of T tokens together in a step."""

    def __init__(self, B, T, seed=0):
        rng = np.random.default_rng(seed)
        z = lambda *n, **k: torch.zeros(n, device="cuda", **k)          # noqa: E731
        half = lambda *n: torch.from_numpy((1 + 0.1 * rng.standard_normal(n)).astype(np.float16)).cuda()      # noqa: E731
        order = lambda n: torch.from_numpy(rng.permutation(n).astype(np.int32)).cuda()                        # noqa: E731
        self.B, self.T, self.rng = B, T, rng
        self.gamma1, self.gamma2 = half(HIDDEN), half(HIDDEN)
        self.order = [order(HIDDEN), order(HIDDEN), order(HIDDEN), order(FFN)]
        self.qkv, self.o, self.gate, self.up, self.down = (weights(n, k, rng) for n, k in (
            ((H + 2 * HKV) * D, HIDDEN), (HIDDEN, HIDDEN), (FFN, HIDDEN), (FFN, HIDDEN), (HIDDEN, FFN)))
        self.rope = atom.atom_rotary_table(torch.tensor([10000.0 ** (-j / PAIRS) for j in range(PAIRS)], dtype=torch.float64, device="cuda"), P)
        self.kc, self.vc = (atom.atom_kv8_cache(B * W, HKV, D, BS) for _ in range(2))
        self.table = torch.full((B, W), -1, dtype=torch.int32, device="cuda")
        self.free = order(B * W)
        self.past, self.new, self.cursor = z(B, dtype=torch.int32), z(B, dtype=torch.int32), z(1, dtype=torch.int32)
        self.positions = z(T, dtype=torch.int32)
        self.x = z(T, HIDDEN, dtype=torch.float16)
        self.attended = z(T, H, D, dtype=torch.float16)

    def inputs(self, new):
        assert len(new) == self.B and sum(new) <= self.T
        pos = np.zeros(self.T, np.int32)
        past = npy(self.past)
        pos[:sum(new)] = np.concatenate([np.arange(p, p + n) for p, n in zip(past, new)])
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        self.positions.copy_(torch.from_numpy(pos))
        self.x.copy_(torch.from_numpy(self.rng.standard_normal((self.T, HIDDEN)).astype(np.float16)))

    def step(self, max_new):
        s = {}
        start, length, slot, cursor = atom.atom_kv_block_map(self.past, self.new, self.table, self.free, self.T, BS, cursor=self.cursor)
        s["qkv"] = atom.atom_w4a16_linear(self.x, self.gamma1, EPS, self.order[0], *self.qkv)
        heads = s["qkv"].view(self.T, H + 2 * HKV, D)
        s["q"], _, _ = atom.atom_rotary_kv8_append(heads[:, :H], heads[:, H:H + HKV], heads[:, H + HKV:], self.kc, self.vc, slot, self.positions, self.rope)
        atom.atom_attention_kv8(s["q"], self.kc, self.vc, self.table, start, length, D ** -0.5, max_new=max_new, out=self.attended)
        s["x1"] = atom.atom_w4a16_linear(self.attended.view(self.T, HIDDEN), None, EPS, self.order[1], *self.o, self.x)
        s["h"] = atom.atom_w4a16_swiglu(s["x1"], self.gamma2, EPS, self.order[2], self.gate, self.up)
        s["x2"] = atom.atom_w4a16_linear(s["h"], None, EPS, self.order[3], *self.down, s["x1"])
        s.update(start=start, length=length, slot=slot, cursor=cursor)
        return s

    def finish(self, s):
        self.past.copy_(s["length"])
        self.cursor.copy_(s["cursor"])


def within(got, want, tol, what):
    off = np.abs(npy(got).astype(np.float64) - want)
    assert np.isfinite(want).all() and (off <= tol).all(), f"{what}: {(off / tol).max():.2f} of the bound"


STEPS = ([40, 3, 0, 17], [1, 1, 35, 1], [1, 1, 1, 1], [1, 30, 1, 0], [1, 1, 1, 1])


def test_every_call_of_a_layer_against_64_bits():
    """Each call by its definition from what the call before it gave; caches bit for bit."""
    s = Server(4, 64)
    for new in STEPS:
        s.inputs(new)
        s.attended.fill_(0.5)                                 # (rows behind the last sequence are left as they were)
        caches = [[npy(t).copy() for t in c] for c in (s.kc, s.vc)]
        r = s.step(max(new))
        w = lambda t: tuple(npy(a) for a in t)                # noqa: E731
        order = [npy(o) for o in s.order]
        within(r["qkv"], *ref.linear(npy(s.x), npy(s.gamma1), EPS, order[0], w(s.qkv)), "qkv")
        heads = npy(r["qkv"]).reshape(s.T, H + 2 * HKV, D)
        turned = ref.turned(heads[:, :H + HKV], npy(s.positions), npy(s.rope))
        assert np.array_equal(npy(r["q"]).view(np.uint16), turned[:, :H].astype(np.float16).view(np.uint16))
        for rows, old, now in ((turned[:, H:], caches[0], s.kc), (heads[:, H + HKV:], caches[1], s.vc)):
            codes, scale = kv8.append(rows, *old, npy(r["slot"]))
            assert np.array_equal(npy(now[0]), codes) and np.array_equal(npy(now[1]), scale)
        want, tol, done = kv8.attention(npy(r["q"]), w(s.kc), w(s.vc), npy(s.table), npy(r["start"]), npy(r["length"]), D ** -0.5)
        assert done[:sum(new)].all() and not done[sum(new):].any()
        off = np.abs(npy(s.attended).astype(np.float64) - want)
        assert (off <= tol)[done].all() and (npy(s.attended)[~done] == 0.5).all()
        within(r["x1"], *ref.linear(npy(s.attended).reshape(s.T, HIDDEN), None, EPS, order[1], w(s.o), npy(s.x)), "o")
        within(r["h"], *ref.swiglu(npy(r["x1"]), npy(s.gamma2), EPS, order[2], w(s.gate), w(s.up)), "gate and up")
        within(r["x2"], *ref.linear(npy(r["h"]), None, EPS, order[3], w(s.down), npy(r["x1"])), "down")
        s.finish(r)


def test_a_prompt_in_parts_fills_the_cache_alike():
    """Queries and caches bit for bit where every step fills whole blocks: a row's sums do not depend on its place in the step."""
    whole, parts = Server(1, 64, seed=3), Server(1, 64, seed=3)
    x = torch.from_numpy(np.random.default_rng(5).standard_normal((64, HIDDEN)).astype(np.float16)).cuda()
    whole.inputs([64])
    whole.x.copy_(x)
    a = whole.step(64)
    for i in range(4):
        parts.inputs([16])
        parts.x[:16] = x[16 * i:16 * i + 16]
        b = parts.step(16)
        assert torch.equal(b["q"][:16], a["q"][16 * i:16 * i + 16])
        parts.finish(b)
    blocks = [npy(s.table)[0, :4] for s in (whole, parts)]
    for c, d in ((whole.kc, parts.kc), (whole.vc, parts.vc)):
        for t, u in zip(c, d):
            assert np.array_equal(npy(t)[blocks[0]], npy(u)[blocks[1]])


def test_a_captured_layer_replays():
    """Captured once, replayed with other lengths, with another server's eager steps between the replays."""
    a, e, other = Server(4, 64, seed=1), Server(4, 64, seed=1), Server(3, 20, seed=2)
    other.inputs([5, 1, 9])
    for s in (a, e):
        s.inputs([1, 1, 1, 1])
        s.step(64)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = a.step(64)
        a.finish(captured)
    for s in (a, e):
        s.past.zero_()
        s.cursor.zero_()
    for new in STEPS:
        for s in (a, e):
            s.rng = np.random.default_rng(sum(new))
            s.attended.fill_(0.25)
            s.inputs(new)
        other.step(9)
        graph.replay()
        eager = e.step(64)
        torch.cuda.synchronize()
        e.finish(eager)
        for n in ("qkv", "q", "x1", "h", "x2"):
            assert torch.equal(captured[n], eager[n]), n
        for c, d in ((a.kc, e.kc), (a.vc, e.vc)):
            assert torch.equal(c[0], d[0]) and torch.equal(c[1], d[1])


def test_two_servers_at_once():
    """Two layers' steps on two streams, launched in turn."""
    servers, new, want = [Server(4, 64, seed=8), Server(2, 24, seed=9)], ([30, 1, 4, 20], [1, 15]), []
    for s, n in zip(servers, new):
        s.inputs(n)
        want.append(s.step(max(n))["x2"].clone())
    streams = [torch.cuda.Stream() for _ in servers]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        got = []
        for s, n, stream in zip(servers, new, streams):
            with torch.cuda.stream(stream):
                got.append(s.step(max(n))["x2"])
    torch.cuda.synchronize()
    for s, n, g, w in zip(servers, new, got, want):
        assert torch.equal(g[:sum(n)], w[:sum(n)])


@pytest.mark.parametrize("gated", [False, True])
def test_a_capture_that_the_allocator_does_not_know_of(gated):
    """A capture begun on the stream itself: the call has to be given its workspace."""
    M = 30
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.standard_normal((M, HIDDEN)).astype(np.float16)).cuda()
    gate, up = weights(FFN, HIDDEN, rng), weights(FFN, HIDDEN, rng)
    need = atom.atom_w4a16_workspace_bytes(M, FFN, HIDDEN, gated=gated, norm=False, index=False)
    assert need > 0
    if gated:
        call = lambda **k: atom.atom_w4a16_swiglu(x, None, EPS, None, gate, up, **k)            # noqa: E731
    else:
        call = lambda **k: atom.atom_w4a16_linear(x, None, EPS, None, *gate, **k)               # noqa: E731
    want, ws = call(), torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(want)
    hip = ctypes.CDLL(next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line))
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        handle, graph, run = ctypes.c_void_p(stream.cuda_stream), ctypes.c_void_p(), ctypes.c_void_p()
        assert hip.hipStreamBeginCapture(handle, 2) == 0      # (relaxed)
        try:
            with pytest.raises(ValueError, match="workspace"):
                call(out=out)
            call(out=out, workspace=ws)
        finally:
            assert hip.hipStreamEndCapture(handle, ctypes.byref(graph)) == 0
        assert hip.hipGraphInstantiate(ctypes.byref(run), graph, None, None, ctypes.c_size_t(0)) == 0
        for _ in range(3):
            out.zero_()
            ws.fill_(0xA5)
            assert hip.hipGraphLaunch(run, handle) == 0
            stream.synchronize()
            assert torch.equal(out, want)
            torch.cuda.synchronize()
        assert hip.hipGraphExecDestroy(run) == 0 and hip.hipGraphDestroy(graph) == 0
