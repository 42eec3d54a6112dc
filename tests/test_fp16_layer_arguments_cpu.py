"""What the entry points of a layer in fp16 activations refuse, decided on the host: pointers that are never followed, and tensors
that claim to be on a GPU (fake tensors have no memory: a call whose arguments pass raises RuntimeError at the device)."""
import ctypes

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import _fp16_layer_ref as ref
import paper_2310_19102_amd as atom
from paper_2310_19102_amd import binding

P, ODD1, ODD2, ODD8 = (ctypes.c_void_p(x) for x in (0x1000, 0x1001, 0x1002, 0x1008))
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


def turn(n_pairs=64, interleaved=0, n_axes=1, axis=()):
    return binding._RotaryDesc(n_pairs, interleaved, n_axes, (ctypes.c_uint8 * 128)(*axis))


@pytest.mark.parametrize("want,changed", [
    (SHAPE, dict(n=0)), (SHAPE, dict(P=-1)), (UNSUPPORTED, dict(n=129)), (UNSUPPORTED, dict(P=2 ** 31)), (UNSUPPORTED, dict(n=128, P=2 ** 25)),
    (0, dict(P=0)), (0, dict(P=0, freq=None)), (NULL, dict(freq=None)), (NULL, dict(table=None)), (ALIGN, dict(freq=ODD2)), (ALIGN, dict(table=ODD8))])
def test_table_refusals(want, changed):
    a = dict(freq=P, n=64, P=100, table=P)
    assert atom.load_library().atom_rotary_table(*{**a, **changed}.values(), None) == want


TURN_REFUSALS = [
    (NULL, dict(r=None)), (SHAPE, dict(r=turn(0))), (SHAPE, dict(r=turn(68))), (SHAPE, dict(r=turn(n_axes=0))), (SHAPE, dict(n_pos=0)),
    (SHAPE, dict(r=turn(axis=[0, 1]))), (SHAPE, dict(r=turn(n_axes=2, axis=[0, 1, 2]))), (SHAPE, dict(r=turn(n_axes=2, axis=[0, 1]), ldp=4)),
    (UNSUPPORTED, dict(r=turn(n_axes=5))), (UNSUPPORTED, dict(r=turn(62))), (UNSUPPORTED, dict(r=turn(interleaved=2))),
    (UNSUPPORTED, dict(n_pos=2 ** 31)), (NULL, dict(pos=None)), (NULL, dict(table=None)), (ALIGN, dict(pos=ODD2)), (ALIGN, dict(table=ODD8))]


@pytest.mark.parametrize("want,changed", [
    *TURN_REFUSALS, (SHAPE, dict(T=-1)), (SHAPE, dict(heads=0)), (SHAPE, dict(D=0)), (SHAPE, dict(ldx=1016)), (SHAPE, dict(ldo=512)),
    (UNSUPPORTED, dict(D=132, ldx=2048, ldo=2048)), (UNSUPPORTED, dict(D=264, ldx=4096, ldo=4096)), (UNSUPPORTED, dict(T=2 ** 26)),
    (UNSUPPORTED, dict(heads=2 ** 24, ldx=2 ** 31, ldo=2 ** 31)), (0, dict(T=0)), (0, dict(T=0, x=None, out=None)),
    (NULL, dict(x=None)), (NULL, dict(out=None)), (ALIGN, dict(x=ODD8)), (ALIGN, dict(out=ODD8)), (ALIGN, dict(ldx=1028)), (ALIGN, dict(ldo=1028))])
def test_rotary_refusals(want, changed):
    a = {**dict(x=P, T=5, ldx=1024, heads=8, D=128, r=turn(), pos=P, ldp=5, table=P, n_pos=99, back=0, out=P, ldo=1024), **changed}
    a["r"] = None if a["r"] is None else ctypes.byref(a["r"])
    assert atom.load_library().atom_rotary(*a.values(), None) == want


@pytest.mark.parametrize("want,changed", [
    *TURN_REFUSALS, (SHAPE, dict(T=-1)), (SHAPE, dict(H=-1)), (SHAPE, dict(Hkv=0)), (SHAPE, dict(D=0)), (SHAPE, dict(n=0)), (SHAPE, dict(ldq=1016)),
    (SHAPE, dict(ldqo=8)), (SHAPE, dict(ldk=511)), (SHAPE, dict(ldv=8)),
    (UNSUPPORTED, dict(D=96, r=turn(32))), (UNSUPPORTED, dict(bs=24)), (UNSUPPORTED, dict(n=2 ** 25)), (UNSUPPORTED, dict(T=2 ** 28)),
    (UNSUPPORTED, dict(T=2 ** 31 - 1)), (0, dict(T=0)), (0, dict(T=0, q=None, k=None)),
    *[(NULL, {k: None}) for k in ("q", "qo", "k", "v", "slot", "kc", "ks", "vc", "vs")],
    *[(ALIGN, {k: ODD8}) for k in ("q", "qo", "k", "v", "kc", "vc")], *[(ALIGN, {k: ODD2}) for k in ("slot", "ks", "vs")],
    (ALIGN, dict(ldq=1028)), (ALIGN, dict(ldqo=1028)), (ALIGN, dict(ldk=516)), (ALIGN, dict(ldv=516))])
def test_rotary_append_refusals(want, changed):
    a = {**dict(q=P, ldq=1024, H=8, qo=P, ldqo=1024, k=P, v=P, T=5, ldk=512, ldv=512, Hkv=4, D=128, r=turn(), pos=P, ldp=5, table=P, n_pos=99,
                slot=P, n=100, bs=64, kc=P, ks=P, vc=P, vs=P), **changed}
    a["r"] = None if a["r"] is None else ctypes.byref(a["r"])
    assert atom.load_library().atom_rotary_kv8_append(*a.values(), None) == want


D = binding._Desc
W4A16 = [
    (NULL, dict(d=None)), (UNSUPPORTED, dict(d=D(1024, 64, 128, 4, 8))), (UNSUPPORTED, dict(d=D(1024, 128, 0, 4, 8))),
    (UNSUPPORTED, dict(d=D(1024, 128, 128, 5, 8))), (SHAPE, dict(d=D(1000, 128, 128, 4, 8))), (SHAPE, dict(d=D(1024, 128, 1024, 4, 8))),
    (UNSUPPORTED, dict(d=D(65536, 128, 128, 4, 8), ldx=65536)), (SHAPE, dict(M=-1)), (SHAPE, dict(N=-1)), (SHAPE, dict(ldx=1016)), (SHAPE, dict(ldy=99)),
    (UNSUPPORTED, dict(M=2 ** 40)), (UNSUPPORTED, dict(M=2 ** 20, N=2 ** 20, ldy=2 ** 20, ldr=2 ** 20)), (0, dict(M=0)), (0, dict(N=0)), (0, dict(M=0, x=None)),
    *[(NULL, {k: None}) for k in ("x", "q4", "q8", "scale", "y")],
    *[(ALIGN, {k: ODD8}) for k in ("x", "gamma", "idx", "q4", "q8")], (ALIGN, dict(scale=ODD1)), (ALIGN, dict(y=ODD1)), (ALIGN, dict(ldx=1028)),
    (WORKSPACE, dict(M=99, ws=None)), (WORKSPACE, dict(M=99, ws_bytes=8)), (ALIGN, dict(M=99, ws=ODD8))]


@pytest.mark.parametrize("want,changed", [*W4A16, (SHAPE, dict(ldr=99)), (ALIGN, dict(res=ODD1))])
def test_linear_refusals(want, changed):
    a = {**dict(x=P, M=5, ldx=1024, gamma=P, eps=0.0, idx=P, d=D(1024, 128, 128, 4, 8), q4=P, q8=P, scale=P, N=100, res=P, ldr=100, y=P, ldy=100,
                ws=P, ws_bytes=1 << 30), **changed}
    a["d"] = None if a["d"] is None else ctypes.byref(a["d"])
    assert atom.load_library().atom_w4a16_linear(*a.values(), None) == want


@pytest.mark.parametrize("want,changed", [*[(w, {k: v for k, v in c.items() if k != "ldr"}) for w, c in W4A16],
                                          *[(NULL, {k: None}) for k in ("u4", "u8", "us")],
                                          (ALIGN, dict(u4=ODD8)), (ALIGN, dict(u8=ODD8)), (ALIGN, dict(us=ODD1))])
def test_swiglu_refusals(want, changed):
    a = {**dict(x=P, M=5, ldx=1024, gamma=P, eps=0.0, idx=P, d=D(1024, 128, 128, 4, 8), q4=P, q8=P, scale=P, u4=P, u8=P, us=P, N=100, y=P, ldy=100,
                ws=P, ws_bytes=1 << 30), **changed}
    a["d"] = None if a["d"] is None else ctypes.byref(a["d"])
    assert atom.load_library().atom_w4a16_swiglu(*a.values(), None) == want


def test_workspace_of_refused_and_plain_calls():
    need = atom.atom_w4a16_workspace_bytes
    assert need(1, 100, 1024) == 0 and need(1, 100, 4096, norm=False, index=False) == 0          # the workgroups lay the row out themselves
    assert need(300, 100, 4096) >= 300 * 4096 * 4 and need(300, 100, 4096, norm=False) >= 300 * 4096 * 2
    for bad in ((-1, 100, 1024), (5, -1, 1024), (0, 100, 1024), (5, 0, 1024), (5, 100, 1000), (2 ** 40, 100, 1024)):
        assert need(*bad) == 0
    assert need(5, 100, 1024, group_size=64) == 0


def fake(*shape, dtype=torch.int32):
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device="cuda")


half = lambda *s: fake(*s, dtype=torch.float16)                          # noqa: E731
single = lambda *s: fake(*s, dtype=torch.float32)                        # noqa: E731
cache = lambda n=9, h=4, bs=64, d=128: (fake(n, h, bs, d, dtype=torch.int8), single(n, h))               # noqa: E731
weights = lambda n=48, k=1024, o=128: (fake(n, (k - o) // 2, dtype=torch.uint8), fake(n, o, dtype=torch.int8), half(n, k // 128))   # noqa: E731

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer")

TURN_TENSORS = [
    (ValueError, dict(positions=fake(6))), (TypeError, dict(positions=fake(5, dtype=torch.int64))), (ValueError, dict(positions=fake(2, 5))),
    (ValueError, dict(positions=fake(2, 5), axis=bytes(63))), (RuntimeError, dict(positions=fake(2, 5), axis=[0, 1] * 32)),
    (RuntimeError, dict(positions=fake(2, 8)[:, :5], axis=bytes(64))), (ValueError, dict(positions=fake(2, 10)[:, ::2], axis=bytes(64))),
    (ValueError, dict(axis=[256] * 64)), (TypeError, dict(axis="a" * 64)),
    (ValueError, dict(table=single(30, 128))), (TypeError, dict(table=half(30, 64, 2))), (ValueError, dict(table=single(30, 2, 64).transpose(1, 2)))]


@pytest.mark.parametrize("error,changed", [
    (RuntimeError, {}), *TURN_TENSORS, (RuntimeError, dict(x=half(5, 24, 128)[:, 8:16])), (ValueError, dict(x=half(5, 1024))),
    (ValueError, dict(x=half(5, 8, 256)[:, :, ::2])), (ValueError, dict(x=half(5, 16, 128)[:, ::2])), (TypeError, dict(x=single(5, 8, 128))),
    (ValueError, dict(x=torch.zeros(5, 8, 128, dtype=torch.float16))), (ValueError, dict(out=half(5, 9, 128))), (TypeError, dict(out=single(5, 8, 128)))])
def test_rotary_tensors(error, changed):
    a = dict(x=half(5, 8, 128), positions=fake(5), table=single(30, 64, 2))
    with pytest.raises(error):
        atom.atom_rotary(**{**a, **changed})


@pytest.mark.parametrize("error,changed", [
    (RuntimeError, {}), *TURN_TENSORS, (RuntimeError, dict(q=None)), (ValueError, dict(q=None, out=half(5, 8, 128))), (ValueError, dict(q=half(4, 8, 128))),
    (ValueError, dict(q=half(5, 8, 64))), (ValueError, dict(k=half(5, 4, 64))), (ValueError, dict(v=half(5, 8, 128))), (ValueError, dict(k_cache=cache(h=8))),
    (ValueError, dict(v_cache=cache(n=8))), (ValueError, dict(k_cache=cache()[:1])), (ValueError, dict(slot=fake(6))), (ValueError, dict(out=half(5, 4, 128)))])
def test_rotary_append_tensors(error, changed):
    a = dict(q=half(5, 8, 128), k=half(5, 4, 128), v=half(5, 4, 128), k_cache=cache(), v_cache=cache(), slot=fake(5), positions=fake(5),
             table=single(30, 64, 2))
    with pytest.raises(error):
        atom.atom_rotary_kv8_append(**{**a, **changed})


LINEAR_TENSORS = [
    (RuntimeError, {}), (ValueError, dict(x=half(5, 1152))), (ValueError, dict(x=half(1024))), (TypeError, dict(x=single(5, 1024))),
    (ValueError, dict(gamma=half(1152))), (ValueError, dict(gamma=half(1, 1024))), (TypeError, dict(gamma=single(1024))),
    (ValueError, dict(reorder_idx=fake(1023))), (TypeError, dict(reorder_idx=fake(1024, dtype=torch.int64))), (ValueError, dict(out=half(5, 47))),
    (ValueError, dict(out=half(48, 5).t())), (TypeError, dict(out=single(5, 48))), (ValueError, dict(group_size=64)),
    (ValueError, dict(workspace=torch.zeros(1 << 20)))]


@pytest.mark.parametrize("error,changed", [
    *LINEAR_TENSORS, (ValueError, dict(residual=half(5, 47))), (ValueError, dict(residual=half(48))), (ValueError, dict(w_q4=weights(47)[0])),
    (ValueError, dict(w_scale=half(48, 9))), (ValueError, dict(w_q8=fake(2, 48, 128, dtype=torch.int8))), (TypeError, dict(w_q4=weights()[0].view(torch.int8)))])
def test_linear_tensors(error, changed):
    w = weights()
    a = dict(x=half(5, 1024), gamma=half(1024), eps=1e-5, reorder_idx=fake(1024), w_q4=w[0], w_q8=w[1], w_scale=w[2])
    with pytest.raises(error):
        atom.atom_w4a16_linear(**{**a, **changed})


@pytest.mark.parametrize("error,changed", [
    *LINEAR_TENSORS, (ValueError, dict(up=weights(47))), (ValueError, dict(gate=weights(48, 1152))), (ValueError, dict(up=weights(48, 1024, 256))),
    (ValueError, dict(gate=weights()[:2])), (TypeError, dict(up=None))])
def test_swiglu_tensors(error, changed):
    a = dict(x=half(5, 1024), gamma=half(1024), eps=1e-5, reorder_idx=fake(1024), gate=weights(), up=weights())
    with pytest.raises(error):
        atom.atom_w4a16_swiglu(**{**a, **changed})


def test_the_reference_on_worked_examples():
    tab = ref.table(8, 4)
    x = np.zeros((1, 1, 16), np.float16)
    x[0, 0, :] = np.arange(16)
    y = ref.turned(x, [2], tab, dtype=np.float64)
    assert np.allclose(y[0, 0, 0], 0 * np.cos(2) - 4 * np.sin(2)) and np.allclose(y[0, 0, 4], 4 * np.cos(2)) and (y[0, 0, 8:] == x[0, 0, 8:]).all()
    y = ref.turned(x, [[2], [3]], tab, axis=[0, 0, 1, 1], interleaved=True, dtype=np.float64)
    assert np.allclose(y[0, 0, 2], 2 * np.cos(0.2) - 3 * np.sin(0.2)) and np.allclose(y[0, 0, 5], 5 * np.cos(0.03) + 4 * np.sin(0.03))
    assert np.isnan(ref.turned(x, [8], tab)[0, 0, :8]).all() and np.isnan(ref.turned(x, [-1], tab)[0, 0, :8]).all()
    codes = ref.codes_of(np.array([[0x7f, 0x80]], np.uint8), np.array([[-128]], np.int8))
    assert codes.tolist() == [[-1, 7, 0, -8, -128]]
