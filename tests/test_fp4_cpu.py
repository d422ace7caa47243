"""4-bit floating point and caches without a GPU: sizes, refusals, and pins of the reference that the GPU tests compare with."""
import ctypes as C
import math

import pytest
import torch

import fp4_reference as ref


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def test_sizes(b):
    assert [b.vptq_fp4_row_bytes(n) for n in (0, 1, 32, 33, 4096, 2 ** 30)] == [0, 16, 16, 32, 2048, 2 ** 29] and b.vptq_fp4_row_bytes(-1) == b.E_SHAPE
    assert [b.vptq_fp4_scale_bytes(*n) for n in ((1, 1), (128, 128), (129, 128), (128, 129), (0, 5), (2 ** 30, 2 ** 30))] == [512, 512, 1024, 1024, 0, 512 * 2 ** 46]
    assert b.vptq_fp4_scale_bytes(-1, 1) == b.vptq_fp4_scale_bytes(1, -1) == b.E_SHAPE
    assert [b.vptq_cache_row_bytes(n, f) for n in (1, 80, 128) for f in ("e4m3", "e2m1")] == [16, 16, 80, 48, 128, 64]
    assert [b.vptq_cache_row_scales(n, f) for n in (1, 80, 129) for f in ("e4m3", "e2m1")] == [1, 1, 1, 3, 2, 5]
    assert b.vptq_cache_row_bytes(0, "e4m3") == b.vptq_cache_row_bytes(b.CACHE_MAX_DIM + 1, "e2m1") == b.vptq_cache_row_scales(0, "e2m1") == b.E_SHAPE
    assert b.lib.vptq_cache_row_bytes(64, b.DTYPE_FP16) == b.lib.vptq_cache_row_scales(64, b.DTYPE_BF16) == b.E_UNSUPPORTED
    with pytest.raises(b.VptqError):
        b.make_cache(1, 1, 1, 0, device="cpu")


def test_linear_queries(b):
    d = b.make_fp4_desc(4096, 4096)
    assert b.vptq_linear_fp4_path(b.make_fp4_desc(0, 4096), 1) == "invalid" and b.lib.vptq_linear_fp4_path(None, 1) == b"invalid"
    # the workspace of 16-bit activations holds the quantized ones, that of e2m1 the status word; a few tokens over a small weight need none
    assert [b.vptq_linear_fp4_workspace_bytes(d, B) for B in (1, 8)] == [0, 0] and b.vptq_linear_fp4_workspace_bytes(d, 9) > 256
    assert b.vptq_linear_fp4_workspace_bytes(b.make_fp4_desc(4096, 4100), 1) > 256 and b.vptq_linear_fp4_workspace_bytes(b.make_fp4_desc(40960, 4096), 1) > 256
    for B in (9, 100, 5000):
        q = b.vptq_linear_fp4_workspace_bytes(b.make_fp4_desc(4096, 4096, "e2m1"), B)
        assert 256 <= q <= b.vptq_linear_fp4_workspace_bytes(d, B) <= 1024 + q + B * 2048 + b.vptq_fp4_scale_bytes(B, 4096)
        assert 1 <= b.vptq_linear_fp4_launches(b.make_fp4_desc(4096, 4096, "e2m1"), B) <= b.vptq_linear_fp4_launches(d, B) <= 2
    for bad, code in ((b.Fp4Desc(0, 1, 0, 0, 0), b.E_SHAPE), (b.Fp4Desc(1, 2 ** 30 + 1, 0, 0, 0), b.E_SHAPE), (b.Fp4Desc(1, 1, b.DTYPE_E4M3, 0, 0), b.E_UNSUPPORTED),
                      (b.Fp4Desc(1, 1, b.DTYPE_FP32, 0, 0), b.E_UNSUPPORTED), (b.Fp4Desc(1, 1, 0, b.DTYPE_E2M1, 0), b.E_UNSUPPORTED), (b.Fp4Desc(1, 1, 0, 0, 1), b.E_UNSUPPORTED)):
        with pytest.raises(b.VptqError) as e:
            b.vptq_linear_fp4_workspace_bytes(bad, 1)
        assert e.value.code == code and b.lib.vptq_linear_fp4_launches(C.byref(bad), 1) == code
    assert b.lib.vptq_linear_fp4_workspace_bytes(C.byref(d), 0) == b.lib.vptq_linear_fp4_workspace_bytes(C.byref(d), 2 ** 30 + 1) == b.E_SHAPE
    assert b.lib.vptq_linear_fp4_workspace_bytes(None, 1) == b.E_NULL


def test_refusals_of_the_c_abi(b):
    """Every one of these returns before anything is launched."""
    L, p = b.lib, 0x1000
    assert L.vptq_fp4_quantize(p, 0, -1, 4, 4, p, p, None) == L.vptq_fp4_quantize(p, 0, 4, 0, 4, p, p, None) == L.vptq_fp4_quantize(p, 0, 4, 4, 3, p, p, None) == b.E_SHAPE
    assert L.vptq_fp4_quantize(p, b.DTYPE_E4M3, 4, 4, 4, p, p, None) == b.E_UNSUPPORTED
    assert L.vptq_fp4_quantize(None, 0, 4, 4, 4, p, p, None) == L.vptq_fp4_quantize(p, 0, 4, 4, 4, None, p, None) == L.vptq_fp4_quantize(p, 0, 4, 4, 4, p, None, None) == b.E_NULL
    assert L.vptq_fp4_quantize(p + 1, 0, 4, 4, 4, p, p, None) == L.vptq_fp4_quantize(p + 2, 2, 4, 4, 4, p, p, None) == L.vptq_fp4_quantize(p, 0, 4, 4, 4, p + 8, p, None) == b.E_ALIGN
    assert L.vptq_fp4_quantize(None, 0, 0, 4, 4, None, None, None) == b.OK
    assert L.vptq_fp4_values(p, p, 4, 0, 0, p, None) == b.E_SHAPE and L.vptq_fp4_values(p, p, 4, 4, b.DTYPE_E4M3, p, None) == b.E_UNSUPPORTED
    assert L.vptq_fp4_values(p, p, 4, 4, 0, None, None) == b.E_NULL and L.vptq_fp4_values(p, p + 4, 4, 4, 0, p, None) == b.E_ALIGN
    assert L.vptq_fp4_values(None, None, 0, 4, 0, None, None) == b.OK
    layer, ptrs = b.make_desc(64, 64, 8, 256, 0, flags=0), b.LayerPtrs(p, p)
    assert L.vptq_dequant_fp4(C.byref(layer), C.byref(ptrs), None, p, None, 0, None) == b.E_NULL
    assert L.vptq_dequant_fp4(C.byref(layer), C.byref(ptrs), p, p + 8, None, 0, None) == b.E_ALIGN
    assert L.vptq_dequant_fp4(C.byref(b.make_desc(64, 2 ** 28, 8, 256, 0, flags=0)), C.byref(ptrs), p, p, None, 0, None) == b.E_SHAPE
    permuted = b.make_desc(64, 64, 8, 256, 0, flags=b.FLAG_COL_PERM)
    assert L.vptq_dequant_fp4(C.byref(permuted), C.byref(b.LayerPtrs(p, p, col_perm=p)), p, p, None, 0, None) == b.E_WORKSPACE
    d, e2m1 = b.make_fp4_desc(64, 64), b.make_fp4_desc(64, 64, "e2m1")

    def linear(desc, x=p, xs=None, w=p, ws=p, out=p, room=p, n=1 << 20):
        return L.vptq_linear_fp4(C.byref(desc), x, xs, 3, w, ws, out, room, n, None)

    assert linear(d, x=None) == linear(d, w=None) == linear(d, ws=None) == linear(d, out=None) == linear(e2m1) == b.E_NULL
    assert linear(d, x=p + 1) == linear(e2m1, x=p + 8, xs=p) == linear(d, w=p + 8) == linear(d, ws=p + 4) == linear(d, out=p + 4) == linear(e2m1, xs=p + 1) == linear(e2m1, xs=p, room=p + 16) == b.E_ALIGN
    assert linear(e2m1, xs=p, room=None) == linear(e2m1, xs=p, n=8) == b.E_WORKSPACE


def cache_desc(b, **other):
    d = dict(n_heads=2, head_dim=64, page_size=16, n_pages=4, n_seqs=1, table_width=3, cache_dtype=b.DTYPE_E4M3, x_dtype=0)
    d.update(other)
    return b.CacheDesc(*d.values())


def test_refusals_of_the_cache(b):
    L, p = b.lib, 0x1000
    ptrs = dict(k=p, v=p, k_scale=p, v_scale=p, table=p, start=p, cu=p)

    def both(desc, code, k_in=p, v_in=p, n=5, **other):
        q = b.CachePtrs(**{**ptrs, **other})
        assert L.vptq_cache_write(C.byref(desc), C.byref(q), k_in, v_in, n, 128, 64, 128, 64, None) == L.vptq_cache_read(C.byref(desc), C.byref(q), k_in, v_in, n, None) == code

    for name, values in dict(n_heads=(0, 4097), head_dim=(0, b.CACHE_MAX_DIM + 1), page_size=(0, 2 ** 30 + 1), n_pages=(0, -1), n_seqs=(-1,), table_width=(-1,)).items():
        for v in values:
            both(cache_desc(b, **{name: v}), b.E_SHAPE)
    both(cache_desc(b), b.E_SHAPE, n=-1)
    both(cache_desc(b, cache_dtype=b.DTYPE_FP16), b.E_UNSUPPORTED)
    both(cache_desc(b, x_dtype=b.DTYPE_E4M3), b.E_UNSUPPORTED)
    for name in ptrs:
        both(cache_desc(b), b.E_NULL, **{name: None})
    both(cache_desc(b), b.E_NULL, k_in=None)
    both(cache_desc(b), b.E_NULL, v_in=None)
    for name in ("k", "v", "k_scale", "v_scale", "table", "start", "cu"):
        both(cache_desc(b), b.E_ALIGN, **{name: p + (8 if name in "kv" else 2)})
    both(cache_desc(b), b.E_ALIGN, k_in=p + 1)
    both(cache_desc(b, x_dtype=2), b.E_ALIGN, v_in=p + 2)
    both(cache_desc(b), b.OK, n=0, k_in=None, v_in=None, table=None)
    both(cache_desc(b, n_seqs=0), b.OK, k_in=None, cu=None)
    assert L.vptq_cache_write(None, None, p, p, 5, 1, 1, 1, 1, None) == L.vptq_cache_read(None, None, p, p, 5, None) == b.E_NULL
    assert L.vptq_cache_write(C.byref(cache_desc(b)), None, p, p, 5, 1, 1, 1, 1, None) == b.E_NULL
    assert L.vptq_cache_write(C.byref(cache_desc(b)), C.byref(b.CachePtrs(**ptrs)), p, p, 5, 128, -64, 128, 64, None) == b.E_SHAPE


def test_tensors_that_are_not_on_a_device_are_refused(b):
    z = torch.zeros
    q, s = z(3, 16, dtype=torch.uint8), z(1, 1, 32, 16, dtype=torch.uint8)
    cache, i = b.make_cache(2, 4, 2, 64, device="cpu"), z(2, dtype=torch.int32)
    for call in (lambda: b.vptq_fp4_quantize(z(3, 32)), lambda: b.vptq_fp4_values(q, s, 32), lambda: b.vptq_linear_fp4(z(3, 32, dtype=torch.float16), q, s),
                 lambda: b.vptq_cache_write(z(1, 2, 64), z(1, 2, 64), *cache, i[:1].view(1, 1), i[:1], i), lambda: b.vptq_cache_read(*cache, i[:1].view(1, 1), i[:1], i, 1, 64)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: b.vptq_fp4_quantize(None), lambda: b.vptq_fp4_values(q, None, 32), lambda: b.vptq_linear_fp4(q, q, None), lambda: b.vptq_cache_write(*[None] * 9),
                 lambda: b.vptq_cache_read(*cache, i, i, i, "1", 64)):
        with pytest.raises(TypeError):
            call()


# ---- pins of the reference -----------------------------------------------------------------------------

def by_hand(block):
    """The rule for one block in plain Python: scale exponent and values."""
    a = max(abs(v) for v in block)
    e = -127
    if a > 0:
        while a >= 7 * math.ldexp(1.0, e):
            e += 1
    grid = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    out = []
    for v in block:
        y = abs(v) / math.ldexp(1.0, e)
        best = min(range(8), key=lambda i: (abs(grid[i] - y), i % 2))
        out.append(math.copysign(grid[best] * math.ldexp(1.0, e), v))
    return e, out


def test_reference_quantization_by_hand():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(40, 70, generator=g) * torch.exp(8 * torch.randn(40, 1, generator=g))
    x[0, :9] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0])
    x[1], x[2, 0], x[3, 0], x[4, 0] = 0, 7.0, 6.9999995, 3.4999998
    x[5, :32] = 1e-45
    v, e = ref.quantize(x)
    for r in range(40):
        for k, c in enumerate(range(0, 70, 32)):
            we, wv = by_hand([float(t) for t in x[r, c:c + 32]])
            assert int(e[r, k]) == we and v[r, c:c + 32].tolist() == wv, (r, k)
    bad, e = ref.quantize(torch.tensor([[1.0] * 32 + [float("inf")] + [1.0] * 31]))
    assert e.tolist() == [[-2 + 0, 128]] and bad[0, :32].eq(1).all() and bad[0, 32:].isnan().all()


def test_reference_layouts_by_hand():
    rows, cols = 200, 300
    bytes_ = torch.arange(rows * 10).remainder(251).to(torch.uint8).view(rows, 10)
    t = ref.scale_tiles(bytes_)
    assert tuple(t.shape) == (2, 3, 32, 16) and torch.equal(ref.scale_rows(t, rows, cols), bytes_)
    assert t[1, 2, 5, 4 * 2 + 1] == bytes_[128 + 64 + 5, 9] and t[0, 0, 31, 12] == bytes_[127, 0] and not t[1, :, 8:, 8:].any() and not t[:, 2, :, 2::4].any()
    q = torch.tensor([[0x21, 0xF7]], dtype=torch.uint8)
    assert ref.code_values(q, 4).tolist() == [[0.5, 1.0, 6.0, -6.0]]
    v = ref.values(torch.tensor([[0x21] + [0] * 15], dtype=torch.uint8), ref.scale_tiles(torch.tensor([[130]], dtype=torch.uint8)), 3)
    assert v.tolist() == [[4.0, 8.0, 0.0]]


def test_reference_places_by_hand():
    i = lambda *v: torch.tensor(v)  # noqa: E731
    assert ref.places(i(4, 9).view(1, 2), i(3), i(1, 4), 4, 10, 6) == [None, (4, 3), (9, 0), (9, 1), None, None]
    assert ref.places(i(4, 9).view(1, 2), i(-1), i(0, 2), 4, 10, 2) == ["gone", (4, 0)]
    assert ref.places(i(4, 10).view(1, 2), i(3), i(0, 7), 4, 10, 7) == [(4, 3)] + ["gone"] * 6
    assert ref.places(i(1, 2, 3).view(3, 1), i(0, 0, 0), i(0, 1, 1, 2), 2, 4, 2) == [(1, 0), (3, 0)]
