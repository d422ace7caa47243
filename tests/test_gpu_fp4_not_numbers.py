"""Blocks of 4-bit operands whose scale byte is 255 (NaN) make NaN of the results that they belong to, and of no others: at columns that end
inside a kernel's step, where the scales that follow in memory are those of the next 128 rows."""
import pytest
import torch

import fp4_reference as ref
from test_gpu_fp4 import check_linear, gen, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def not_numbers(rows, cols, some):
    """(scale bytes, the same with 255 in the blocks `some` = [(row, block)], the rows that have none of these)."""
    good = torch.full((rows, ref.up(cols, 32)), 125, dtype=torch.uint8, device="cuda")
    bad, keep = good.clone(), torch.ones(rows, dtype=torch.bool, device="cuda")
    for r, k in some:
        bad[r, k], keep[r] = 255, False
    return ref.scale_tiles(good), ref.scale_tiles(bad), keep


# one, three, five (the last with eight columns), seven tiles of 128 columns: an odd number; and two, four for comparison
COLS = [128, 384, 520, 640, 896, 3200, 256, 512]


@pytest.mark.parametrize("B", [1, 8, 9, 40, 300])
@pytest.mark.parametrize("N", COLS)
def test_a_weights_block(b, N, B):
    g = gen(N + B)
    M, last = 700, ref.up(N, 32) - 1
    w, _ = ref.random_weight(M, N, g, "cuda")
    x = torch.randn(B, N, generator=g, device="cuda").bfloat16()
    # a row's first blocks in the second, third and sixth tile of rows, and its last block in each
    good, bad, keep = not_numbers(M, N, [(128 + 5, 0), (128 + 37, 1), (256 + 64, 2), (256 + 127, 3), (640, 0), (650, last), (699, last), (255, last)])
    clean = check_linear(b, x, w, good, "fp32", N, ref.quantize(x)[0])
    y = b.vptq_linear_fp4(x, w, bad, out_dtype="fp32")
    assert y[:, ~keep].isnan().all() and same(y[:, keep], clean[:, keep])
    q, s = b.vptq_fp4_quantize(x)
    clean = b.vptq_linear_fp4(q, w, good, x_scale=s, out_dtype="fp32")
    y = b.vptq_linear_fp4(q, w, bad, x_scale=s, out_dtype="fp32")
    assert y[:, ~keep].isnan().all() and same(y[:, keep], clean[:, keep])


# (pairs of CTAs and single ones, wide tiles and narrow ones, columns split over clusters)
@pytest.mark.parametrize("M,N,B", [(8192, 384, 2048), (4096, 640, 1000), (28672, 128, 300), (37888, 384, 100), (18944, 640, 16), (300, 8320, 16), (2000, 5760, 30), (1000, 2176, 500)])
def test_a_weights_block_and_many_tokens(b, M, N, B):
    g = gen(M)
    last = ref.up(N, 32) - 1
    w, _ = ref.random_weight(M, N, g, "cuda")
    q, s = ref.random_weight(B, N, g, "cuda")
    good, bad, keep = not_numbers(M, N, [(128 + 5, 0), (128 + 37, 1), (256 + 10, 2), (256 + 43, 3), (M - 1, last), (M - 40, 0)])
    clean = check_linear(b, q, w, good, "fp32", N, ref.values(q, s, N), s)
    y = b.vptq_linear_fp4(q, w, bad, x_scale=s, out_dtype="fp32")
    assert y[:, ~keep].isnan().all() and same(y[:, keep], clean[:, keep])


@pytest.mark.parametrize("N", COLS)
def test_a_tokens_block(b, N):
    g = gen(N)
    M, B, last = 300, 300, ref.up(N, 32) - 1
    w, ws = ref.random_weight(M, N, g, "cuda")
    q, _ = ref.random_weight(B, N, g, "cuda")
    good, bad, keep = not_numbers(B, N, [(128 + 5, 0), (128 + 37, 1), (256 + 10, 2), (256 + 43, 3), (255, last), (299, last)])
    clean = b.vptq_linear_fp4(q, w, ws, x_scale=good, out_dtype="fp32")
    y = b.vptq_linear_fp4(q, w, ws, x_scale=bad, out_dtype="fp32")
    assert y[~keep].isnan().all() and same(y[keep], clean[keep])


@pytest.mark.parametrize("N", [128, 640])
def test_a_weights_block_of_the_next_128_rows(b, N):
    """Every row of the second tile of rows is NaN: the first tile's results stay what they are, for every number of tokens."""
    g = gen(N)
    w, _ = ref.random_weight(256, N, g, "cuda")
    good, bad, keep = not_numbers(256, N, [(128 + r, k) for r in range(128) for k in range(4)])
    for B in range(1, 18):
        x = torch.randn(B, N, generator=g, device="cuda").half()
        clean, y = (b.vptq_linear_fp4(x, w, s, out_dtype="fp32") for s in (good, bad))
        assert clean.isfinite().all() and y[:, 128:].isnan().all() and same(y[:, :128], clean[:, :128])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_largest_magnitudes(b, dtype):
    """From 3.5 * 2^126 on a value becomes 2^128, which FP32 and BF16 do not have; what is smaller reads back as a number."""
    x = torch.zeros(4, 64, device="cuda", dtype=dtype)
    x[0, 0], x[1, 0], x[2, 0], x[3, 5] = 3.5 * 2.0 ** 126, 3.46875 * 2.0 ** 126, torch.finfo(dtype).max, -torch.finfo(dtype).max
    q, s = b.vptq_fp4_quantize(x)
    assert [int(v) for v in ref.scale_rows(s, 4, 64)[:, 0]] == [253, 252, 253, 253]
    want = torch.zeros(4, 64, dtype=torch.float64, device="cuda")
    want[0, 0], want[1, 0], want[2, 0], want[3, 5] = 2.0 ** 128, 6 * 2.0 ** 125, 2.0 ** 128, -2.0 ** 128
    assert torch.equal(ref.values(q, s, 64), want)
    cache, i = b.make_cache(1, 4, 1, 64, "e2m1"), lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    b.vptq_cache_write(x.view(4, 1, 64), x.view(4, 1, 64), *cache, i(0).view(1, 1), i(0), i(0, 4))
    for out, t in (("fp32", torch.float32), ("bf16", torch.bfloat16)):
        assert torch.equal(b.vptq_fp4_values(q, s, 64, out), want.float().to(t))
        assert all(torch.equal(r.view(4, 64), want.float().to(t)) for r in b.vptq_cache_read(*cache, i(0).view(1, 1), i(0), i(0, 4), 4, 64, out))
