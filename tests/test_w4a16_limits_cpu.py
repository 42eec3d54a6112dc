"""The largest W4A16 calls: a launch has fewer than 2^32 threads in a dimension, whatever number of parts of K the call is shared out in, and what could need more is refused by
its sizes, on the host.  Calls on the accepted side stop at a null pointer, which is asked for after the sizes."""
import ctypes
import random

import pytest

import paper_2310_19102_amd as atom
from _w4a16_shapes import shape
from paper_2310_19102_amd import binding

P = ctypes.c_void_p(0x1000)
NULL, UNSUPPORTED = 1, 3


def status(M, N, K, O=128, gated=False):
    d = binding._Desc(K, 128, O, 4, 8)
    L = atom.load_library()
    if gated:
        return L.atom_w4a16_swiglu(None, M, K, None, 0.0, None, ctypes.byref(d), P, P, P, P, P, P, N, P, N, P, 0, None)
    return L.atom_w4a16_linear(None, M, K, None, 0.0, None, ctypes.byref(d), P, P, P, N, None, 0, P, N, P, 0, None)


def threads(M, N, K, O, gated):
    """Of the call's largest launch: a row to 1024 threads, a tile's part to 512, 256 results of a join to 256."""
    kept, _, NT, wide, parts = shape(M, N, K, O, gated, True, True)
    tiles = -(-N // (128 if gated else 256)) * -(-M // (32 * wide)) if wide else min(-(-N // (16 * NT)), 512)
    return max(M * 1024, tiles * parts * 512, -(-M * N // 256) * 256 if parts > 1 else 0)


@pytest.mark.parametrize("M,N,K,gated,want", [
    (2 ** 22 - 1, 128, 256, False, NULL), (2 ** 22, 128, 256, False, UNSUPPORTED), (2 ** 22 - 1, 129, 256, False, UNSUPPORTED), (2 ** 22 - 32, 129, 256, False, NULL),        # blocks of 32 rows and 128 outputs: 2^18 - 2
    (2 ** 21 - 32, 256, 256, True, NULL), (31, 128 * (2 ** 18 - 1), 256, True, NULL), (33, 128 * (2 ** 17 - 1), 256, True, NULL), (33, 128 * 2 ** 17, 256, True, UNSUPPORTED),
    (16, 2 ** 25 - 128, 256, False, NULL), (16, 2 ** 25 - 127, 256, False, UNSUPPORTED),
    (1, 2 ** 17 - 1, 32768, False, NULL), (63, 2 ** 24 - 128, 256, False, NULL), (63, 2 ** 24 - 127, 256, False, UNSUPPORTED),
    (2 ** 15, 2 ** 15, 256, False, UNSUPPORTED), (2 ** 15, 2 ** 15 - 1, 256, False, UNSUPPORTED), (2 ** 15 - 64, 2 ** 15 - 64, 256, False, NULL)])
def test_the_largest_calls(M, N, K, gated, want):
    assert status(M, N, K, gated=gated) == want
    if want == NULL:
        assert threads(M, N, K, 128, gated) < 2 ** 32


def test_no_accepted_call_has_a_larger_launch():
    rng = random.Random(11)
    accepted = 0
    for _ in range(20000):
        M, K = round(2 ** rng.uniform(0, 23)), 128 * round(2 ** rng.uniform(1, 8))
        N = max(1, min(round(2 ** rng.uniform(0, 26)), round(2 ** (31 * rng.random() ** 0.2)) // M))
        gated = rng.random() < 0.5
        if status(M, N, K, gated=gated) == NULL:
            accepted += 1
            assert threads(M, N, K, 128, gated) < 2 ** 32, (M, N, K, gated)
    assert 5000 < accepted < 20000
