"""The pieces of the scores' gradient cover all of it once, up to the largest sizes that the entry point takes (no GPU)."""
from __future__ import annotations

import pytest

from paper_2503_20591_b200 import binding as nb, build as lib_build

MOST = nb.NBOS_POLICY_MAX_ROWS


@pytest.fixture(scope="module", autouse=True)
def lib():
    lib_build.build()
    return nb.load_library()


@pytest.mark.parametrize("values", [1, 2])
@pytest.mark.parametrize("groups,rows,hosts", [(1, 1, 1), (1, 255, 257), (7, 1000, 3000), (5, 1500, 40001), (1, 70003, 4099), (1, 4099, 70001), (65535, 32768, 3),
                                               (2, MOST // 2, 5), (1, MOST, 64), (1, MOST - 1, 64), (1, MOST, 1), (1, MOST, 4097), (1, MOST, nb.NBOS_MAX_HOSTS),
                                               (1, MOST // 3, 100000), (1, nb.NBOS_MAX_HOSTS, nb.NBOS_MAX_HOSTS)])
def test_pieces_cover_all(groups, rows, hosts, values):
    pieces, entries, largest = nb.nbos_probe_towers_pieces(groups, rows, hosts, values)
    assert entries == groups * rows * hosts and pieces >= 1
    # about 512 MB, or one tile's 256 rows or hosts of the longer side
    assert largest <= max(512 << 20, 0) + 2 * values * 256 * max(min(rows, hosts) + 63, 64)


def test_refusals():
    for bad in ((0, 1, 1, 2), (65536, 1, 1, 2), (1, 0, 1, 2), (1, MOST + 1, 1, 2), (2, MOST, 1, 2), (1, 1, 0, 2), (1, 1, 1 << 21, 2), (1, 1, 1, 0), (1, 1, 1, 3)):
        with pytest.raises(nb.NbosError):
            nb.nbos_probe_towers_pieces(*bad)
