"""Sizes that a launch of the 8-bit building blocks cannot take are refused (no GPU: a call that is not refused reaches the runtime)."""
import ctypes
import os

import pytest
import torch

from paper_2508_17588_amd import binding as B


@pytest.mark.skipif(torch.cuda.is_available(), reason="the buffers are made up")
def test_widest_weight():
    if not os.path.exists(B.LIB_PATH):
        from paper_2508_17588_amd.build import build
        build(verbose=False)
    lib = B.load_library()
    buffers = [ctypes.c_void_p(i << 36) for i in (1, 2, 3)]

    def rc(columns, block_rows):
        return lib.hero_quantize_fp8(buffers[0], 0, 1, columns, block_rows, buffers[1], buffers[2], None)
    # 2^24 blocks of 128 columns at 256 threads each are 2^32 threads
    assert rc((1 << 31) - 112, 128) == rc((1 << 31) - 16, 128) == B.HERO_ERR_SHAPE and b"2^31" in lib.hero_last_error()
    for columns, block_rows in (((1 << 31) - 128, 128), ((1 << 31) - 16, 1)):
        assert rc(columns, block_rows) not in (B.HERO_ERR_SHAPE, B.HERO_ERR_INVALID_ARG)
