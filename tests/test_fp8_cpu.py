"""8-bit floating point operators: sizes, paths and every refusal of a call, without a GPU."""
import ctypes as C

import pytest
import torch

import fp8_reference as ref
from paper_2409_17066_b200 import build as vbuild


@pytest.fixture(scope="module")
def b():
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def test_reference_rounding_is_the_types_own():
    # every finite e4m3 value, and the midpoints between neighbours, against torch's own conversion
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    every = every[torch.isfinite(every)].sort().values.unique()
    mid = (every[1:] + every[:-1]) / 2
    for v in (every, mid, torch.randn(10000, dtype=torch.float64) * 50):
        v = v.clamp(-448, 448)
        assert torch.equal(ref.e4m3(v), v.float().to(torch.float8_e4m3fn).double())


def test_row_bytes(b):
    assert [b.vptq_fp8_row_bytes(n) for n in (0, 1, 15, 16, 17, 4096, 2 ** 31 - 1)] == [0, 16, 16, 16, 32, 4096, 2 ** 31]
    assert b.vptq_fp8_row_bytes(-1) == b.E_SHAPE


def test_quantize_refusals(b):
    f, p = b.lib.vptq_fp8_quantize, 0x1000
    assert f(p, 0, 4, 0, 8, 1, p, p, None) == b.E_SHAPE
    assert f(p, 0, -1, 8, 8, 1, p, p, None) == b.E_SHAPE
    assert f(p, 0, 4, 8, 7, 1, p, p, None) == b.E_SHAPE             # rows would overlap
    assert f(p, 0, 4, 8, 8, 64, p, p, None) == b.E_SHAPE
    assert f(p, b.DTYPE_E4M3, 4, 8, 8, 1, p, p, None) == b.E_UNSUPPORTED
    assert f(None, 0, 4, 8, 8, 1, p, p, None) == b.E_NULL
    assert f(p, 0, 4, 8, 8, 1, None, p, None) == b.E_NULL
    assert f(p, 0, 4, 8, 8, 1, p, None, None) == b.E_NULL
    assert f(p, 0, 4, 8, 8, 1, p + 8, p, None) == b.E_ALIGN
    assert f(p, 0, 4, 8, 8, 1, p, p + 4, None) == b.E_ALIGN
    assert f(p + 1, 0, 4, 8, 8, 1, p, p, None) == b.E_ALIGN
    assert f(p + 2, b.DTYPE_FP32, 4, 8, 8, 1, p, p, None) == b.E_ALIGN
    assert f(None, 0, 0, 8, 8, 1, None, None, None) == b.OK         # no rows: nothing to do


def test_dequant_fp8_refusals(b):
    f, p = b.lib.vptq_dequant_fp8, 0x1000
    d = b.make_desc(64, 64, 8, 256)
    ptrs = b.LayerPtrs(p, p, None, None, None, None, p, p)
    assert b.lib.vptq_dequant_fp8_workspace_bytes(C.byref(d)) == 0
    assert f(None, C.byref(ptrs), p, p, None, 0, None) == b.E_NULL
    assert f(C.byref(d), C.byref(b.LayerPtrs()), p, p, None, 0, None) == b.E_NULL
    assert f(C.byref(d), C.byref(ptrs), None, p, None, 0, None) == b.E_NULL
    assert f(C.byref(d), C.byref(ptrs), p + 8, p, None, 0, None) == b.E_ALIGN
    bad = b.make_desc(64, 64, 8, 70000)
    assert f(C.byref(bad), C.byref(ptrs), p, p, None, 0, None) == b.E_SHAPE
    perm = b.make_desc(64, 100, 8, 256, flags=b.FLAG_SCALE_BIAS | b.FLAG_COL_PERM)
    pp = b.LayerPtrs(p, p, None, None, None, None, p, p, p)
    need = b.lib.vptq_dequant_fp8_workspace_bytes(C.byref(perm))
    assert need >= 400
    assert f(C.byref(perm), C.byref(pp), p, p, None, 0, None) == b.E_WORKSPACE
    assert f(C.byref(perm), C.byref(pp), p, p, p, need - 1, None) == b.E_WORKSPACE
    assert f(C.byref(perm), C.byref(pp), p, p, p + 16, need, None) == b.E_ALIGN


def test_sizes_beyond_the_counters_are_refused(b):
    p = 0x1000
    assert b.lib.vptq_fp8_quantize(p, 0, 2 ** 31 - 1, 1, 1, 1, p, p, None) == b.E_SHAPE
    assert b.lib.vptq_fp8_quantize(p, 0, 1, 2 ** 30 + 1, 2 ** 31, 1, p, p, None) == b.E_SHAPE
    # (an index's bit in its row is counted in 32 bits)
    ptrs = b.LayerPtrs(p, p, None, None, None, None, p, p)
    wide = b.make_desc(8, 2 ** 28, 8, 65536)
    assert b.lib.vptq_dequant_fp8(C.byref(wide), C.byref(ptrs), p, p, None, 0, None) == b.E_SHAPE


def test_linear_fp8_refusals(b):
    f, p = b.lib.vptq_linear_fp8, 0x1000
    d = b.make_fp8_desc(64, 64, "e4m3", "fp16")
    call = lambda d, B=1, x=p, xs=p, w=p, ws=p, out=p: f(C.byref(d), x, xs, B, w, ws, out, None, 0, None)  # noqa: E731
    assert f(None, p, p, 1, p, p, p, None, 0, None) == b.E_NULL
    for hole in ("x", "xs", "w", "ws", "out"):
        assert call(d, **{hole: None}) == b.E_NULL, hole
        assert call(d, **{hole: p + 8}) == b.E_ALIGN, hole
    assert call(d, B=0) == b.E_SHAPE
    for M, N in ((0, 64), (64, 0), (-1, 64), (2 ** 31 - 1, 64), (64, 2 ** 31 - 1)):
        assert call(b.make_fp8_desc(M, N)) == b.E_SHAPE
        assert b.lib.vptq_linear_fp8_workspace_bytes(C.byref(b.make_fp8_desc(M, N)), 1) == b.E_SHAPE
    bad = b.make_fp8_desc(64, 64)
    bad.x_dtype = b.DTYPE_FP32
    assert call(bad) == b.E_UNSUPPORTED
    bad = b.make_fp8_desc(64, 64)
    bad.out_dtype = b.DTYPE_E4M3
    assert call(bad) == b.E_UNSUPPORTED
    assert call(b.make_fp8_desc(64, 64, flags=b.FLAG_SCALE_BIAS)) == b.E_UNSUPPORTED
    assert b.vptq_linear_fp8_path(bad, 1) == "invalid"
    assert b.vptq_linear_fp8_path(d, 8) == "fp8_decode" and b.vptq_linear_fp8_path(d, 9) == "fp8_tcgen05"
    h = b.make_fp8_desc(100, 300, "bf16", "fp32")
    assert b.vptq_linear_fp8_workspace_bytes(h, 8) == 0 and b.vptq_linear_fp8_workspace_bytes(d, 9) == 256
    need = b.vptq_linear_fp8_workspace_bytes(h, 9)
    assert need >= 256 + 9 * (304 + 4 * 3)                          # status word, e4m3 rows, scales
    assert f(C.byref(h), p, None, 9, p, p, p, None, 0, None) == b.E_WORKSPACE
    assert f(C.byref(h), p, None, 9, p, p, p, p, need - 1, None) == b.E_WORKSPACE
    assert f(C.byref(h), p, None, 9, p, p, p, p + 16, need, None) == b.E_ALIGN
    assert [b.vptq_linear_fp8_launches(x, B) for x in (d, h) for B in (8, 9)] == [1, 1, 1, 2]
    assert b.vptq_linear_fp8_launches(d, 1) == 1 and b.vptq_linear_fp8_launches(d, 0) == b.E_SHAPE


def test_host_tensors_are_refused_before_any_call(b):
    x, w, s = torch.zeros(2, 64, dtype=torch.float16), torch.zeros(64, 64, dtype=torch.float8_e4m3fn), torch.ones(1, 1)
    with pytest.raises(AssertionError):
        b.vptq_fp8_quantize(x)
    with pytest.raises(AssertionError):
        b.vptq_linear_fp8(x, w, s)
    with pytest.raises(TypeError):
        b.vptq_linear_fp8(None, w, s)
    with pytest.raises(b.VptqError):
        b.vptq_fp8_quantize(x, 64)


def test_moe_fp8_refusals(b):
    f, p = b.lib.vptq_moe_fp8, 0x1000
    names = [n for n, _ in b.MoePtrs._fields_]
    ptrs = b.MoePtrs(*[p] * 7)
    d = b.make_moe_desc(256, 128, 8, 2)
    size = lambda d, T=1: b.lib.vptq_moe_fp8_workspace_bytes(C.byref(d), T)  # noqa: E731
    call = lambda d, T=1, ptrs=ptrs, x=p, out=p, ws=p, n=1 << 30: f(C.byref(d), C.byref(ptrs), x, T, out, ws, n, None)  # noqa: E731
    assert f(None, C.byref(ptrs), p, 1, p, p, 1 << 30, None) == b.E_NULL and f(C.byref(d), None, p, 1, p, p, 1 << 30, None) == b.E_NULL
    assert call(d, x=None) == b.E_NULL and call(d, out=None) == b.E_NULL
    assert call(d, x=p + 2) == b.E_ALIGN and call(d, out=p + 2) == b.E_ALIGN and call(d, ws=p + 16) == b.E_ALIGN
    for i, name in enumerate(names):
        for value, code in ((None, b.E_NULL), (p + 4, b.E_ALIGN)):
            args = [p] * 7
            args[i] = value
            assert call(d, ptrs=b.MoePtrs(*args)) == code, name
    need = size(d, 3)
    assert need >= 3 * 2 * 128 * 4 and size(d, 4) > need
    assert call(d, T=3, ws=None) == b.E_WORKSPACE and call(d, T=3, n=need - 1) == b.E_WORKSPACE
    for T in (0, -1, b.MOE_MAX_TOKENS + 1):
        assert call(d, T=T) == b.E_SHAPE and size(d, T) == b.E_SHAPE
    for bad in ((0, 128, 8, 2), (256, 0, 8, 2), (256, 128, 0, 2), (256, 128, 8, 0), (256, 128, 8, 9), (256, 128, b.MOE_MAX_EXPERTS + 1, 2),
                (256, 128, 64, b.MOE_MAX_TOP + 1), (1 << 24, 128, 64, 2), (256, 1 << 24, 64, 2)):
        assert call(b.make_moe_desc(*bad)) == b.E_SHAPE, bad
    assert call(b.make_moe_desc(256, 128, 8, 2, flags=b.FLAG_SCALE_BIAS)) == b.E_UNSUPPORTED
    assert call(b.make_moe_desc(256, 128, 8, 2, x_dtype="fp32")) == b.E_UNSUPPORTED
    bad = b.make_moe_desc(256, 128, 8, 2)
    bad.out_dtype = b.DTYPE_E4M3
    assert call(bad) == b.E_UNSUPPORTED
    x = torch.zeros(1, 256, dtype=torch.float16)
    with pytest.raises(AssertionError):
        b.vptq_moe_fp8(x, x, *[x[None]] * 6, 2)
