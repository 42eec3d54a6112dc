"""What the paged 8-bit KV cache's entry points refuse, decided on the host: pointers that are never followed, and tensors that
claim to be on a GPU (fake tensors have no memory: a call whose arguments pass raises RuntimeError at the device)."""
import ctypes

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import _kv8_ref as ref
import paper_2310_19102_amd as atom

P, ODD2, ODD8 = (ctypes.c_void_p(x) for x in (0x1000, 0x1002, 0x1008))
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


@pytest.mark.parametrize("want,changed", [
    (SHAPE, dict(B=-1)), (SHAPE, dict(W=0)), (SHAPE, dict(W=-1)), (SHAPE, dict(T=-1)), (SHAPE, dict(n_free=-1)),
    (UNSUPPORTED, dict(bs=0)), (UNSUPPORTED, dict(bs=8)), (UNSUPPORTED, dict(bs=48)), (UNSUPPORTED, dict(bs=256)),
    (UNSUPPORTED, dict(B=16385)), (UNSUPPORTED, dict(T=2 ** 31 - 1)), (UNSUPPORTED, dict(W=2 ** 24 + 1)),
    (UNSUPPORTED, dict(B=16384, W=2 ** 17)),
    (NULL, dict(past=None)), (NULL, dict(new=None)), (NULL, dict(table=None)), (NULL, dict(start=None)), (NULL, dict(length=None)),
    (NULL, dict(slot=None)), (NULL, dict(free=None)), (NULL, dict(B=0, start=None)),
    *[(ALIGN, {k: ODD2}) for k in ("past", "new", "free", "cursor", "table", "start", "length", "slot", "cursor_out")]])
def test_block_map_refusals(want, changed):
    a = dict(past=P, new=P, B=4, bs=64, free=P, n_free=9, cursor=None, table=P, W=8, T=12, start=P, length=P, slot=P, cursor_out=P)
    assert atom.load_library().atom_kv_block_map(*{**a, **changed}.values(), None) == want


@pytest.mark.parametrize("want,changed", [
    (SHAPE, dict(T=-1)), (SHAPE, dict(Hkv=0)), (SHAPE, dict(D=0)), (SHAPE, dict(n=0)), (SHAPE, dict(ldk=511)), (SHAPE, dict(ldv=8)),
    (UNSUPPORTED, dict(D=96, ldk=1024, ldv=1024)), (UNSUPPORTED, dict(bs=24)), (UNSUPPORTED, dict(n=2 ** 25)),
    (UNSUPPORTED, dict(n=2 ** 24, Hkv=40, ldk=1 << 13, ldv=1 << 13)), (UNSUPPORTED, dict(T=2 ** 30)), (0, dict(T=0)),
    (0, dict(T=0, k=None, slot=None)),
    *[(NULL, {k: None}) for k in ("k", "v", "slot", "kc", "ks", "vc", "vs")],
    *[(ALIGN, {k: ODD8}) for k in ("k", "v", "kc", "vc")], *[(ALIGN, {k: ODD2}) for k in ("slot", "ks", "vs")],
    (ALIGN, dict(ldk=516)), (ALIGN, dict(ldv=514))])
def test_append_refusals(want, changed):
    a = dict(k=P, v=P, T=5, ldk=512, ldv=512, Hkv=4, D=128, slot=P, n=100, bs=64, kc=P, ks=P, vc=P, vs=P)
    assert atom.load_library().atom_kv8_append(*{**a, **changed}.values(), None) == want


ATTENTION = dict(q=P, T=5, ldq=1024, B=3, H=8, Hkv=4, D=128, max_new=5, start=P, length=P, table=P, W=99, n=100, bs=64, kc=P, ks=P,
                 vc=P, vs=P, sm=0.1, out=P, ldo=1024, ws=P, ws_bytes=1 << 30)


@pytest.mark.parametrize("want,changed", [
    (SHAPE, dict(T=-1)), (SHAPE, dict(B=-1)), (SHAPE, dict(H=0)), (SHAPE, dict(Hkv=0)), (SHAPE, dict(Hkv=3)), (SHAPE, dict(D=0)),
    (SHAPE, dict(max_new=-1)), (SHAPE, dict(W=0)), (SHAPE, dict(n=0)), (SHAPE, dict(ldq=1023)), (SHAPE, dict(ldo=512)),
    (UNSUPPORTED, dict(D=32)), (UNSUPPORTED, dict(bs=20)), (UNSUPPORTED, dict(W=2 ** 24 + 1)), (UNSUPPORTED, dict(n=2 ** 25)),
    (UNSUPPORTED, dict(T=2 ** 28)), (UNSUPPORTED, dict(sm=-0.1)), (UNSUPPORTED, dict(sm=float("nan"))), (UNSUPPORTED, dict(sm=float("inf"))),
    (UNSUPPORTED, dict(B=2 ** 29, max_new=1)), (UNSUPPORTED, dict(B=2 ** 30)),
    (0, dict(T=0)), (0, dict(B=0, W=0)), (0, dict(max_new=0)), (0, dict(T=0, q=None, out=None, ws=None)),
    *[(NULL, {k: None}) for k in ("q", "start", "length", "table", "kc", "ks", "vc", "vs", "out")],
    *[(ALIGN, {k: ODD8}) for k in ("q", "kc", "vc", "out", "ws")], *[(ALIGN, {k: ODD2}) for k in ("start", "length", "table", "ks", "vs")],
    (ALIGN, dict(ldq=1028)), (ALIGN, dict(ldo=1026)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=4))])
def test_attention_refusals(want, changed):
    lib = atom.load_library()
    assert atom.atom_attention_kv8_workspace_bytes(5, 3, 8, 4, 128, 5, 99, 64) > 4
    assert lib.atom_attention_kv8(*{**ATTENTION, **changed}.values(), None) == want


def test_workspace_of_refused_and_of_unsplit_calls():
    need = atom.atom_attention_kv8_workspace_bytes
    assert need(1, 1, 32, 32, 128, 1, 16, 64) > 0
    assert need(4096, 4096, 32, 32, 128, 1, 16, 64) == 0                 # enough workgroups as it is
    assert need(1, 1, 32, 32, 128, 1, 2, 64) == 0                       # too few keys to share out
    # uncut in workgroups of 16, 8 and 4 wavefronts as long as the longest sequence costs less than a merge
    for B, Hkv, D, bs, W, cut in ((1, 32, 128, 64, 8, False), (1, 32, 128, 64, 16, True), (8, 32, 128, 64, 33, False), (8, 32, 128, 64, 60, True),
                                  (1, 4, 64, 16, 70, False), (1, 4, 64, 16, 150, True), (64, 8, 128, 64, 16, False), (64, 8, 128, 64, 60, True),
                                  (100, 8, 128, 128, 1, False), (100, 8, 128, 128, 20, True)):
        assert (need(B, B, Hkv, Hkv, D, 1, W, bs) > 0) == cut, (B, Hkv, D, bs, W)
    for bad in ((1, 1, 32, 5, 128, 1, 16, 64), (1, 1, 32, 32, 96, 1, 16, 64), (1, 1, 32, 32, 128, 1, 16, 60), (-1, 1, 32, 32, 128, 1, 16, 64),
                (0, 1, 32, 32, 128, 1, 16, 64), (1, 0, 32, 32, 128, 1, 16, 64), (1, 1, 32, 32, 128, 0, 16, 64)):
        assert need(*bad) == 0


def fake(*shape, dtype=torch.int32):
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device="cuda")


half = lambda *s: fake(*s, dtype=torch.float16)                          # noqa: E731
cache = lambda n=9, h=4, bs=64, d=128: (fake(n, h, bs, d, dtype=torch.int8), fake(n, h, dtype=torch.float32))   # noqa: E731

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer")


@pytest.mark.parametrize("error,changed", [
    (RuntimeError, {}), (ValueError, {0: fake(4, 1)}), (TypeError, {0: fake(4, dtype=torch.int64)}), (ValueError, {1: fake(5)}),
    (ValueError, {2: fake(3, 8)}), (ValueError, {2: fake(32)}), (ValueError, {2: fake(8, 4).t()}), (ValueError, {3: fake(3, 3)}),
    (ValueError, {0: torch.zeros(4, dtype=torch.int32)}), (TypeError, {4: 1.5}), (ValueError, {5: 2 ** 32 + 64})])
def test_block_map_tensors(error, changed):
    a = [fake(4), fake(4), fake(4, 8), fake(30), 12, 64]
    with pytest.raises(error):
        atom.atom_kv_block_map(*[changed.get(i, x) for i, x in enumerate(a)])


@pytest.mark.parametrize("error,changed", [
    (RuntimeError, {}), (RuntimeError, {0: half(5, 12, 128)[:, 4:8], 1: half(5, 12, 128)[:, 8:]}), (ValueError, {0: half(5, 4, 64)}),
    (ValueError, {0: half(5, 512), 1: half(5, 512)}), (ValueError, {0: half(5, 4, 256)[:, :, ::2], 1: half(5, 4, 128)}),
    (ValueError, {0: half(5, 8, 128)[:, ::2]}), (TypeError, {1: half(5, 4, 128).float()}), (ValueError, {2: cache(h=8)}),
    (ValueError, {3: cache(n=8)}), (ValueError, {2: cache()[:1]}), (ValueError, {2: (cache()[0], fake(9, 5, dtype=torch.float32))}),
    (TypeError, {2: (cache()[0], half(9, 4))}), (ValueError, {4: fake(6)}), (TypeError, {4: fake(5, dtype=torch.int64)})])
def test_append_tensors(error, changed):
    a = [half(5, 4, 128), half(5, 4, 128), cache(), cache(), fake(5)]
    with pytest.raises(error):
        atom.atom_kv8_append(*[changed.get(i, x) for i, x in enumerate(a)])


@pytest.mark.parametrize("error,changed", [
    (RuntimeError, {}), (ValueError, {0: half(5, 8, 64)}), (ValueError, {0: half(5, 8, 256)[:, :, ::2]}), (ValueError, {1: cache(n=8)}),
    (ValueError, {3: fake(24)}), (ValueError, {4: fake(3)}), (ValueError, {5: fake(4)}), (ValueError, {7: -1}), (TypeError, {6: "x"}),
    (TypeError, {4: fake(4, dtype=torch.int64)})])
def test_attention_tensors(error, changed):
    a = [half(5, 8, 128), cache(), cache(), fake(3, 8), fake(4), fake(3), 0.1, 5]
    with pytest.raises(error):
        atom.atom_attention_kv8(*[changed.get(i, x) for i, x in enumerate(a)])


def test_the_definitions_agree_on_a_worked_example():
    """Two requests on blocks of sixteen tokens: tables, slots and codes by hand."""
    table = np.array([[7, -1, -1], [-1, -1, -1]], np.int32)
    start, length, slot, cursor, table = ref.block_map([15, 0], [2, 17], table, [4, 2, 9], 20, 16)
    assert start.tolist() == [0, 2, 19] and length.tolist() == [17, 17] and cursor.tolist() == [3]
    assert table.tolist() == [[7, 4, -1], [2, 9, -1]]
    assert slot.tolist() == [127, 64, *range(32, 48), 144, -1]
    codes, scale = np.zeros((2, 1, 16, 2), np.int8), np.zeros((2, 1), np.float32)
    codes, scale = ref.append(np.array([[[1.27, -0.5]]], np.float16), codes, scale, [16])
    assert scale[1, 0] == np.float32(np.float16(1.27)) / np.float32(127) and codes[1, 0, 0].tolist() == [127, -50]
    codes, scale = ref.append(np.array([[[2.54, 0.01]]], np.float16), codes, scale, [17])
    # 127 / 2 and -50 / 2 of the doubled scale; fp16(0.01) / (fp16(2.54) / 127) = 0.010002 / 0.019993 = 0.5003, which is 1
    assert codes[1, 0, :2].tolist() == [[64, -25], [127, 1]]
