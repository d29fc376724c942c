"""Calls of the operators that are larger than a launch."""
import paper_2506_01151_amd as zf


def test_quantize_refuses_more_blocks_than_a_launch_takes():
    """Blocks of 128 rows are a workgroup each: 2^24 - 1 of 256 threads at most.  (Refused before anything is read: the addresses are none.)"""
    L = zf.load_library()
    for rows, cols in (((1 << 31) - 1, 1), (1 << 20, 1 << 18), (1 << 31 >> 7, 1 << 24)):
        assert L.zf_quantize_blocks(4096, 0, rows, cols, cols, 128, 4096, 4096, 0, None) == zf.ZF_ERR_INVALID_ARG and b"split the rows" in L.zf_last_error(), (rows, cols)
