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


@pytest.mark.parametrize("hidden,inner,experts,top,T", [(256, 128, 8, 2, 1), (333, 200, 5, 5, 3), (2048, 1024, 64, 8, 1), (4096, 14336, 8, 2, 32), (16, 16, 1, 1, 32)])
def test_the_workspace_of_the_experts_has_room_for_its_parts(b, hidden, inner, experts, top, T):
    """The list of experts, h in e4m3 with its scales, and a copy of x in e4m3 with its scales for each of the 37 clusters that a device
    of 148 SMs (the one counted with where there is none) has room for."""
    pitch = lambda n: -(-n // 16) * 16  # noqa: E731
    pairs, most = T * top, b.MOE_MAX_TOKENS * b.MOE_MAX_TOP
    plan = 16 + most * (4 + 2 + 2 + 2 * 8)
    parts = [plan, pairs * pitch(inner), pairs * 4 * -(-inner // 128), 37 * T * pitch(hidden), 37 * T * 4 * -(-hidden // 128)]
    need = b.vptq_moe_fp8_workspace_bytes(b.make_moe_desc(hidden, inner, experts, top), T)
    assert need == sum(-(-n // 256) * 256 for n in parts)


def test_the_workspace_of_the_product_has_room_for_its_parts(b):
    for M, N, B in ((100, 300, 9), (64, 8192, 2048), (5, 16, 129)):
        for x_type, parts in (("e4m3", []), ("bf16", [B * 4 * -(-N // 128), B * -(-N // 16) * 16])):
            need = b.vptq_linear_fp8_workspace_bytes(b.make_fp8_desc(M, N, x_type), B)
            assert 256 + sum(parts) <= need < 256 + sum(parts) + 256
