"""Registers and LDS of the kernels of the 4-bit cache, of appends and of the
selection of pages: none spills, and as many workgroups share a CU as they are
laid out for."""
import re

import pytest

from .test_registers import kernels

NAMES = ("append_rotated", "page_bounds", "read_rows4", "nibble_rows", "nibble_tiles", "page_scores", "select_pages",
         "picked_rows", "picked_tiles",
         "new_bounds")
KERNELS = {n: (m[1], k) for n, k in kernels().items() if (m := re.search(r"\d+(" + "|".join(NAMES) + r")I", n))}


def test_every_kernel_is_there():
    count = dict.fromkeys(NAMES, 0)
    for name, _ in KERNELS.values():
        count[name] += 1
    assert count == {"append_rotated": 32, "page_bounds": 4, "read_rows4": 4, "nibble_rows": 10, "nibble_tiles": 8,
                     "page_scores": 4, "select_pages": 3, "picked_rows": 4, "picked_tiles": 2,
                     "new_bounds": 4}


# fp32, d = 128, 256 rows: a few words outside the loop over tiles
SPILLS = {("f", "128", "8"): 5}


@pytest.mark.parametrize("name", sorted(KERNELS))
def test_spills(name):
    m = re.search(r"nibble_tilesI([tf])Li(\d+)ELi(\d)E", name)
    most = SPILLS.get(m.groups(), 0) if m else 0
    k = KERNELS[name][1]
    assert k[".vgpr_spill_count"] <= most and k[".sgpr_spill_count"] == 0
    assert k[".private_segment_fixed_size"] <= 8 * most


def waves(k):
    """Waves of a SIMD that the vector registers leave room for."""
    return 512 // (-(-(k[".vgpr_count"] + k.get(".agpr_count", 0)) // 8) * 8)


@pytest.mark.parametrize("name", sorted(n for n, (x, _) in KERNELS.items() if x.startswith("nibble")))
def test_workgroups_to_a_cu(name):
    """Four of 32-key decode tiles, two of 64; two of 128 rows in bf16, one of
    256 rows and of fp32."""
    k = KERNELS[name][1]
    m = re.search(r"nibble_(rows|tiles)I([tf])Li\d+E(?:\w*?ELi(\d\d)E|Li(\d)E)", name)
    if m[1] == "rows":
        wgs, per = (4, 4) if m[3] == "32" else (2, 4)
    else:
        per = int(m[4])
        wgs = 2 if (m[2], per) == ("t", 4) else 1
    assert waves(k) >= wgs * per // 4 and wgs * k[".group_segment_fixed_size"] <= 160 << 10
