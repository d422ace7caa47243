"""Arguments of the 8-bit floating point operators that are refused before anything runs, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2409_17066_b200 import build as vbuild


@pytest.fixture(scope="module")
def b():
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def test_a_workspace_in_host_memory_is_refused(b):
    # (the kernels would write to it)
    p = 0x1000
    desc = b.make_desc(64, 100, 8, 256, flags=b.FLAG_SCALE_BIAS | b.FLAG_COL_PERM)
    ptrs = b.LayerPtrs(p, p, None, None, None, None, p, p, p)
    need = b.lib.vptq_dequant_fp8_workspace_bytes(C.byref(desc))
    with pytest.raises(AssertionError, match="workspace"):
        b.vptq_dequant_fp8(desc, ptrs, torch.zeros(need, dtype=torch.uint8))


def test_a_layer_elsewhere_is_refused(b):
    # (its addresses are nothing that the current device's kernels may read)
    desc = b.make_desc(64, 64, 8, 256)
    streams = [torch.zeros(1 << 14, dtype=torch.uint8) for _ in range(4)]
    idx, table, scale, bias = (t.data_ptr() for t in streams)
    with pytest.raises(AssertionError, match="current device"):
        b.vptq_dequant_fp8(desc, b.LayerPtrs(idx, table, None, None, None, None, scale, bias))
    out = b.make_desc(64, 64, 8, 256, 0, 64, 8, 16)
    with pytest.raises(AssertionError, match="current device"):
        b.vptq_dequant_fp8(out, b.LayerPtrs(None, None, None, None, idx, table, scale, bias))
