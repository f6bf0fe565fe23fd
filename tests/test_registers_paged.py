"""Registers and LDS of the compiled kernels of the paged cache: what they
spill, and that two workgroups of the attention share a CU."""
import re

import pytest

from .test_registers import kernels

# kernel, element type (t: bf16), head dim -> vector and scalar registers that
# it may spill.  Scalar registers go to the lanes of vector registers, not to
# memory.  The two vector registers of fp32 decode at d = 128 are spilled
# outside its loop over tiles.
SPILLS = {("attend_rows", "f", 128, "NoSeqs"): (2, 0), ("attend_rows", "f", 128, "PagedSeqs"): (0, 140),
          ("attend_rows", "f", 64, "PagedSeqs"): (0, 70), ("attend_rows", "t", 128, "PagedSeqs"): (0, 30),
          ("attend_rows", "t", 64, "PagedSeqs"): (0, 30), ("attend_tiles", "t", 128, ""): (0, 10),
          ("attend_shared", "f", 128, ""): (0, 20)}


def paged_kernels():
    """(kernel, element type, head dim, sequences) -> metadata."""
    out = {}
    for name, k in kernels().items():
        m = re.search(r"\d+(attend_rows|attend_shared|attend_tiles|paged_join|join_weights|prefill_weights|"
                      r"evict_select|evict_copy|evict_move)(I([tf])?Li(\d+)E(.*NoSeqs|.*PagedSeqs|Li\dE)?)?", name)
        if m:
            seqs = next((s for s in ("NoSeqs", "PagedSeqs") if m[1] == "attend_rows" and s + "E" in name), "")
            out[name] = ((m[1], m[3] or "t", int(m[4] or 0), seqs), k)
    return out


KERNELS = paged_kernels()


def test_every_kernel_is_there():
    count = {}
    for (kernel, *_), _k in KERNELS.values():
        count[kernel] = count.get(kernel, 0) + 1
    assert count == {"attend_rows": 8, "attend_shared": 4, "attend_tiles": 2, "paged_join": 8, "join_weights": 4,
                     "prefill_weights": 4, "evict_select": 2, "evict_copy": 1, "evict_move": 1}


@pytest.mark.parametrize("name", sorted(KERNELS))
def test_spills(name):
    key, k = KERNELS[name]
    vector, scalar = SPILLS.get(key, (0, 35 if key[0] == "join_weights" else 0))
    assert k[".vgpr_spill_count"] <= vector and k[".sgpr_spill_count"] <= scalar, key
    assert k[".private_segment_fixed_size"] <= 8 * vector, key     # bytes of scratch a thread


@pytest.mark.parametrize("name", sorted(n for n, (key, _) in KERNELS.items() if key[0].startswith("attend")))
def test_two_workgroups_to_a_cu(name):
    """256 registers for each of two waves per SIMD, half of 160 KB of LDS."""
    _, k = KERNELS[name]
    assert k[".vgpr_count"] + k.get(".agpr_count", 0) <= 256 and k[".group_segment_fixed_size"] <= 80 << 10
