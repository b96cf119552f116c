"""The built code of the products with a step per group and of the attention over the 4-bit cache, as the compiler lists it: distances
that it cannot see to itself because inline assembly is part of them, and what their counted waits take for granted.  CPU only
(hipcc cross-compiles)."""
import os

import pytest

from test_listing import HIPCC, instructions, listing, loads_behind_m0, too_close


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
@pytest.mark.parametrize("source", ["sq_w4a16_grouped.hip", "sq_tree_attention.hip"])
def test_listing(source, tmp_path):
    lines = listing(source, tmp_path)
    found, readers = too_close(lines)
    assert readers > 100 and not found, found[:4]
    found, loads = loads_behind_m0(lines)
    assert loads > 10 and not found, found[:4]
    assert not [text for text, _ in instructions(lines) if text.startswith("v_pk_") and text.split()[0].endswith("_f32")]
    # kernels that load into LDS wait for a number of loads: registers that went to memory would be among them
    function, uses_lds_loads, spills = "", set(), set()
    for line in lines:
        if line.startswith("_ZN") and ":" in line:
            function = line.split(":")[0]
        if "global_load_lds" in line:
            uses_lds_loads.add(function)
        if line.strip().startswith("scratch_"):
            spills.add(function)
    assert uses_lds_loads and not uses_lds_loads & spills
