"""Rotary positions of many tokens of one, two and three heads, bit for bit as in test_gpu_rotary.py: fewer heads than a lane would take of more."""
import pytest

import _fp16_layer_ref as ref
import paper_2310_19102_amd as atom
from test_gpu_rotary import case, gpu, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,heads,D,R,axes", [
    (8199, 1, 128, 128, 1), (30011, 1, 64, 32, 3), (196700, 1, 128, 64, 1), (4201, 2, 128, 128, 1), (9001, 2, 64, 64, 2), (98400, 2, 128, 96, 1), (5003, 3, 128, 128, 1)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_bits(T, heads, D, R, axes, interleaved):
    x, pos, tab, axis = case(T, heads, D, R, axes, interleaved, seed=2)
    want = ref.turned(x, pos, tab, axis, interleaved, interleaved)
    xd, pd, td = gpu(x, pos, tab)
    same(atom.atom_rotary(xd, pd, td, axis, interleaved, interleaved), want)
    atom.atom_rotary(xd, pd, td, axis, interleaved, interleaved, out=xd)
    same(xd, want)
