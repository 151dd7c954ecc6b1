"""Workgroups of a CU, kernel by kernel, of the small updates and of the pairs' products with three steps in shared memory: what their launches count on, from the registers
and the shared memory in the notes of the built library's code objects (CPU)."""
import re

import pytest

from test_host_matrix_registers import fit, kernels  # noqa: F401

# k_small by its bytes: three workgroups are let in by registers (four by shared memory), two by shared memory, one
SMALL = {("f32", 1, 40832): 3, ("bf16", 1, 40832): 3, ("f32", 1, 81792): 2, ("bf16", 1, 81792): 2, ("f32", 2, 163712): 1, ("bf16", 2, 163712): 1, ("f32", 5, 163712): 1, ("bf16", 5, 163712): 1}
# kKinds of csrc/qoda_orthogonal.hip: {(side, steps in shared memory): workgroups}
PAIRS = {(64, 2): 4, (64, 3): 2, (96, 3): 1, (128, 2): 2, (256, 2): 1}


def test_small_updates(kernels):  # noqa: F811
    found = {}
    for name, (registers, scratch, shared) in kernels.items():
        m = re.search(r"k_smallI(f|NS_4bf16E)Li(\d+)ELi(\d+)EEEv", name)
        if m:
            found["f32" if m.group(1) == "f" else "bf16", int(m.group(2)), int(m.group(3))] = fit(8, registers, shared)
            assert scratch == 0 and shared >= int(m.group(3))
    assert found.keys() == SMALL.keys()
    for key, a_cu in SMALL.items():
        assert found[key] >= a_cu, (key, found[key])


def test_tiles_of_pairs(kernels):  # noqa: F811
    found = {}
    for name, (registers, scratch, shared) in kernels.items():
        m = re.search(r"k_pair_productILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d)EEEv", name)
        if m:
            side, across, wm, wn, steps = map(int, m.groups())
            found[side, steps] = fit(wm * wn, registers, shared)
            assert across == side and scratch == 0 and shared == steps * 2 * side * 128
    assert found.keys() == PAIRS.keys()
    for key, a_cu in PAIRS.items():
        assert found[key] >= a_cu, (key, found[key])


@pytest.mark.parametrize("waves,registers,shared,want", [(8, 64, 40896, 4), (8, 80, 40896, 3), (8, 96, 40896, 2), (4, 128, 1, 4), (4, 129, 1, 3), (4, 256, 1, 2), (8, 80, 163776, 1)])
def test_what_fits(waves, registers, shared, want):
    assert fit(waves, registers, shared) == want
