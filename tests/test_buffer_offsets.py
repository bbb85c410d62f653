"""Loads and stores through sized buffer resources carry their whole offset where the bounds are checked (the vector and
immediate parts); a scalar offset comes on top, unchecked."""
import os
import re

import pytest

from paper_2609_35140_amd import asm_hazards as H
from paper_2609_35140_amd import build as B


@pytest.mark.parametrize("source", ["uattn_decode_mx.hip"])
def test_no_scalar_offsets(source):
    seen = 0
    for ln in H.assembly(os.path.join(B.CSRC, source)).splitlines():
        m = re.match(r"\s+buffer_(?:load|store)\w*\s+(.*)", ln)
        if m:
            seen += 1
            assert m.group(1).split(",")[3].split()[0] == "0", ln.strip()  # data, vector offset, resource, scalar offset
    assert seen > 0
