"""Steps without tokens: empty rows have no heads that could lie apart, so whatever strides an empty slice has it is taken, and nothing is written."""
import pytest
import torch

import paper_2310_19102_amd as atom

pytestmark = pytest.mark.gpu


def empties(heads, D):
    r = torch.zeros((6, D, 2 * heads), dtype=torch.float16, device="cuda")
    return [r[:0, :heads].new_empty((0, heads, D)), r.transpose(1, 2)[:0, ::2], torch.zeros((3, 2 * heads, D), dtype=torch.float16, device="cuda")[3:, ::2]]


@pytest.mark.parametrize("which", range(3))
def test_every_entry_point_that_takes_rows(which):
    D, bs = 64, 16
    q, k = empties(4, D)[which], empties(2, D)[which]
    caches = [atom.atom_kv8_cache(3, 2, D, bs) for _ in range(2)]
    for codes, scale in caches:
        codes.fill_(5)
        scale.fill_(0.5)
    none, tab = torch.empty(0, dtype=torch.int32, device="cuda"), torch.zeros((9, 8, 2), device="cuda")
    atom.atom_kv8_append(k, k, *caches, none)
    out, kc, vc = atom.atom_rotary_kv8_append(q, k, k, *caches, none, none, tab)
    assert out.shape == (0, 4, D) and kc is caches[0] and vc is caches[1]
    assert atom.atom_rotary(q, none, tab).shape == (0, 4, D)
    start = torch.zeros(2, dtype=torch.int32, device="cuda")
    got = atom.atom_attention_kv8(q, *caches, torch.zeros((1, 2), dtype=torch.int32, device="cuda"), start, start[:1], 0.1, max_new=1)
    assert got.shape == (0, 4, D)
    for codes, scale in caches:
        assert bool((codes == 5).all()) and bool((scale == 0.5).all())
