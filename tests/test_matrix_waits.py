"""The wait states between a matrix instruction and the reads of its result that the compiler left out (planted cases; the
kernels themselves are checked with the inline assembly's)."""
from paper_2609_35140_amd import asm_hazards as H

MFMA = "\tv_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[12:15], 0\n"


def _fn(body):
    return "kernel:\n" + body + "\ts_endpgm\n"


def test_straight_line():
    read = "\tv_maximum3_f32 v20, v1, v7, v7\n"
    assert len(H.scan_matrix(_fn(MFMA + "\ts_nop 5\n" + read))) == 1
    assert H.scan_matrix(_fn(MFMA + "\ts_nop 7\n" + read)) == []
    assert H.scan_matrix(_fn(MFMA + "\tv_mov_b32_e32 v20, v3\n")) == []
    assert len(H.scan_matrix(_fn(MFMA + "\tds_write_b128 v30, v[4:7]\n"))) == 1
    assert len(H.scan_matrix(_fn(MFMA + "\tds_read_b128 v[30:33], v5 offset:64\n"))) == 1
    assert H.scan_matrix(_fn(MFMA + "\tds_read_b128 v[4:7], v30\n")) == []     # (overwritten, not read)


def test_branch_around_a_body_that_waits_long_enough():
    body = "".join(f"\tv_cndmask_b32_e64 v{30 + i}, v{30 + i}, v20, s[4:5]\n" for i in range(16))
    text = _fn(MFMA + "\ts_cbranch_scc1 .LBB0_2\n" + body + ".LBB0_2:\n\tv_maximum3_f32 v20, v1, v7, v7\n")
    found = H.scan_matrix(text)
    assert len(found) == 1 and "with 1 wait states" in found[0]
    assert H.scan_matrix(text.replace("\ts_cbranch", "\ts_nop 7\n\ts_cbranch")) == []


def test_another_result_in_between():
    """The register is written again before the read: the matrix instruction's result is not the one read."""
    assert H.scan_matrix(_fn(MFMA + "\tv_mov_b32_e32 v7, 0\n\tv_maximum3_f32 v20, v1, v7, v7\n")) == []
