"""Kernels whose registers are planned to the last one keep all they hold in registers: no spills, no scratch memory."""
import os

import pytest

from paper_2609_35140_amd import asm_hazards as H
from paper_2609_35140_amd import build as B


@pytest.mark.parametrize("source,kernels", [("uattn_decode_mx.hip", 70), ("uattn_kv_mx.hip", 36)])
def test_no_scratch(source, kernels):
    found = H.resources(H.assembly(os.path.join(B.CSRC, source)))
    assert len(found) >= kernels
    for name, r in found.items():
        assert r["vgpr_spill_count"] == 0 and r["private_segment_fixed_size"] == 0, name
