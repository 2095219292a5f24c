"""How many values may hold an entry of the towers' gradient: refusals, and the layout of the struct that says so."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2503_20591_b200 import binding as nb, build as lib_build, policy

FAKE = 1 << 20   # an address that is aligned and never read


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return nb.load_library()


@pytest.mark.parametrize("values", [-1, 3, 1 << 30])
def test_refused(lib, values):
    packed = nb._TOWERS.pack(FAKE, FAKE, 8, 64, 512, 64, 6400, 2, 100, 64, nb.NBOS_BF16, 0, 0, values)
    fields = nb.nbos_towers(FAKE, FAKE, 8, 64, 512, 64, 6400, 2, 100, 64, nb.NBOS_BF16, None, None, values)
    for towers in (packed, ctypes.byref(fields)):
        for status in (lib.nbos_policy_towers(towers, FAKE, FAKE, 3, 3, 1.0, FAKE, None, None),
                       lib.nbos_policy_towers_backward(towers, FAKE, FAKE, 3, 3, 1.0, FAKE, None, 1.0, FAKE, 64, 512, FAKE, 64, 6400, None)):
            assert status == nb.NBOS_ERR_INVALID_ARG and "gradient_values" in nb.nbos_last_error_detail()


def test_the_two_layouts_are_one():
    assert nb._TOWERS.size == ctypes.sizeof(nb.nbos_towers)
    numbers = (1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 2)
    assert bytes(nb.nbos_towers(*numbers)) == nb._TOWERS.pack(*numbers)


@pytest.mark.parametrize("values", [0, 3, "2", None])
def test_autograd_form_refuses(values):
    v = torch.zeros(2, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="gradient_values"):
        policy.tower_distill_loss(v, v, torch.zeros(2, 1, dtype=torch.int32), gradient_values=values)
