"""Which kernels the W4A16 calls launch: the rule in _w4a16_shapes.py is the library's, as far as the workspace shows it, and the sizes of the GPU tests
reach every one of them."""
import random

import paper_2310_19102_amd as atom
import test_gpu_w4a16
import test_gpu_w4a16_many_outputs as many
from _w4a16_shapes import ALL, kernels, shape


def parts_bytes(M, N, K, O, gated, norm, index):
    """The workspace of a call behind its laid out rows: the parts' sums."""
    kept, _, _, wide, parts = shape(M, N, K, O, gated, norm, index)
    return parts * M * N * (8 if gated else 4) if parts > 1 else 0


def laid_out_bytes(M, N, K, O, gated, norm, index):
    kept, _, _, wide, _ = shape(M, N, K, O, gated, norm, index)
    units = (K + O) // 128 * (2 if norm else 1)
    return 0 if kept else units * M * 256 if not wide else -(-M // (32 * wide)) * wide * units * 8192


def back_bytes(M, N, K, O, gated, norm, index):
    """What takes the rows' powers of two back, behind a norm."""
    return -(-M // 64) * 256 if norm and not shape(M, N, K, O, gated, norm, index)[0] else 0


def test_the_rule_is_the_library_s():
    rng = random.Random(3)
    for _ in range(3000):
        M, K = round(2 ** rng.uniform(0, 8)), 128 * round(2 ** rng.uniform(1.01, 8))
        N, O = round(2 ** rng.uniform(0, 16.5)), 128 * rng.choice([1, 1, 1, 2, min(3, K // 128 - 1)])
        if O >= K:
            continue
        gated, norm, index = (rng.random() < 0.5 for _ in range(3))
        got = atom.atom_w4a16_workspace_bytes(M, N, K, n_outlier=O, gated=gated, norm=norm, index=index)
        args = (M, N, K, O, gated, norm, index)
        assert got == laid_out_bytes(*args) + back_bytes(*args) + parts_bytes(*args), args


def test_every_kernel_is_tested():
    seen = set()
    for M, N, K, O in test_gpu_w4a16.SIZES:
        for norm, index in ((True, True), (False, False), (False, True), (True, False)):
            seen.update(kernels(M, N, K, O, False, norm, index))
        for norm, index in ((True, True), (False, False), (False, True)):
            seen.update(kernels(M, N, K, O, True, norm, index))
    before = set(seen)
    for M, N, K in many.SIZES:
        for norm, index, _ in many.WAYS:
            for gated in (False, True):
                seen.update(kernels(M, N, K, 128, gated, norm, index))
    assert seen == ALL
    assert {k for k in ALL - before if k[0] == "few"} >= {("few", 4, False, 2, False, False), ("few", 2, True, 1, True, False)}


def test_workgroups_with_several_tiles_in_turn():
    """Two a compute unit (256 of them) at most."""
    for norm, gated in ((n, g) for n in (False, True) for g in (False, True)):
        assert any(-(-N // (16 * shape(M, N, K, 128, gated, norm)[2])) > 512 and not shape(M, N, K, 128, gated, norm)[0] for M, N, K in many.SIZES)
