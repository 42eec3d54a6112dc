"""The largest calls of the paged 8-bit KV cache: a launch has fewer than 2^32 threads, and what would need more is refused by its sizes, on the host.
Calls on the accepted side stop at a null pointer, which is asked for after the sizes."""
import ctypes

import pytest

import paper_2310_19102_amd as atom

P = ctypes.c_void_p(0x1000)
NULL, UNSUPPORTED = 1, 3


@pytest.mark.parametrize("bs,T,Hkv,want", [
    (64, 2 ** 27 - 64, 4, NULL), (64, 2 ** 27 - 63, 4, UNSUPPORTED), (64, 2 ** 27, 4, UNSUPPORTED),        # 64 tokens to a workgroup of 256 threads and head
    (16, 2 ** 27 - 64, 4, NULL), (16, 2 ** 27, 4, UNSUPPORTED), (32, 1, 2 ** 23 - 1, NULL), (32, 1, 2 ** 23, UNSUPPORTED),
    (64, 255, 131586, NULL), (128, 255, 131587, UNSUPPORTED), (64, 1, 2 ** 25 - 2, NULL), (64, 1, 2 ** 25 - 1, UNSUPPORTED)])    # a wavefront for each
def test_append(bs, T, Hkv, want):
    D = 64
    assert atom.load_library().atom_kv8_append(None, None, T, Hkv * D, Hkv * D, Hkv, D, P, 1, bs, P, P, P, P, None) == want


@pytest.mark.parametrize("B,T,max_new,H,Hkv,W,want", [
    (65535, 65535, 1, 256, 256, 1, NULL), (65536, 65536, 1, 256, 256, 1, UNSUPPORTED), (65536, 65536, 1, 256, 256, 4096, UNSUPPORTED),
    (65535, 2 ** 18, 4, 512, 256, 2, NULL), (65536, 2 ** 18, 4, 512, 256, 2, UNSUPPORTED), (2 ** 14 - 1, 2 ** 14, 1, 2 ** 13, 1024, 1, NULL),
    (2 ** 14, 2 ** 14, 1, 2 ** 13, 1024, 1, UNSUPPORTED),
    (65536, 70000, 1, 8, 1, 1, NULL), (65537, 70000, 1, 8, 1, 1, UNSUPPORTED)])            # lengths that every workgroup scans
def test_attention(B, T, max_new, H, Hkv, W, want):
    D = 128
    assert atom.load_library().atom_attention_kv8(None, T, H * D, B, H, Hkv, D, max_new, P, P, P, W, 100, 64, P, P, P, P, ctypes.c_float(0.1), P,
                                                  H * D, P, 0, None) == want
