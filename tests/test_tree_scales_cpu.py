"""Scales whose product with log2(e) is no finite float are refused, like infinities and NaN."""
import ctypes
import os

import numpy as np
import pytest

from paper_2601_01513_amd import binding as B


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4028234e38, float(np.nextafter(np.float32(2.0 ** 127), np.float32(np.inf))),
                                   float("inf"), float("-inf"), float("nan")])
def test_scales_past_the_range(scale):
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libvsr.so not built (python -m paper_2601_01513_amd.build)")
    lib = B.load_library()
    p = B.VsrPages(n_seqs=1, n_pages=4, page_size=16, max_pages=2, table=1 << 20, table_stride=2,
                   len=1 << 21, held=1 << 22, refs=None)
    h = [ctypes.byref(B.VsrHeads(i << 24, 1, 64, 64)) for i in range(1, 5)]
    # (No rows: what is not refused has nothing to do.)
    args = [B.VSR_F32, 64, 0, 1 << 23, *h[:3], None, 0, 0]
    assert lib.vsr_tree_attention(ctypes.byref(p), *args, scale, h[3], None, None, 0, None) == B.VSR_EINVAL
    assert "scale" in lib.vsr_last_error(None).decode()
    for fine in (2.0 ** 127, -2.0 ** 127, 0.0, 1e-40):
        assert lib.vsr_tree_attention(ctypes.byref(p), *args, fine, h[3], None, None, 0, None) == B.VSR_OK
