"""4-bit floating point operators against their definitions in 64 bits."""
import pytest
import torch

import fp4_reference as ref
from oracle import oracle
from paper_2409_17066_b200 import synth

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def same(a, b):
    """Equal bit for bit (NaNs too)."""
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def check_quantized(q, scale, x):
    rows, cols = x.shape
    want, e = ref.quantize(x)
    assert q.dtype == scale.dtype == torch.uint8 and tuple(q.shape) == (rows, 16 * ref.up(cols, 32))
    assert torch.equal(scale, ref.scale_tiles((e + 127).to(torch.uint8)))            # with zeros where there are no rows and blocks
    got = ref.values(q, scale, cols)
    assert ((got == want) | (got.isnan() & want.isnan())).all()
    assert torch.equal(torch.signbit(got)[want == 0], torch.signbit(x.double())[want == 0])
    codes = torch.stack([q & 15, q >> 4], dim=-1).flatten(1)
    assert not codes[:, cols:].any()                                                   # pad codes are zeros


def check_linear(b, x, w, w_scale, out_dtype, N, x_values, x_scale=None, **more):
    y = b.vptq_linear_fp4(x, w, w_scale, x_scale=x_scale, out_dtype=out_dtype, **more)
    want, bound = ref.linear(x_values, ref.values(w, w_scale, N), TYPES[out_dtype])
    assert y.dtype == TYPES[out_dtype] and tuple(y.shape) == tuple(want.shape)
    off = (y.double() - want).abs()
    assert (off <= bound).all(), (float((off / bound).max()), float(off.max()))
    return y


# ---- quantization -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (2, 31), (3, 32), (127, 33), (128, 128), (129, 1000), (300, 333), (1, 7), (2000, 776), (5000, 1032), (37, 130)])
def test_quantize(b, rows, cols, dtype):
    g = gen(rows * 1000 + cols)
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(3 * torch.randn(rows, 1, generator=g, device="cuda"))
    x = x.to(TYPES[dtype])
    check_quantized(*b.vptq_fp4_quantize(x), x)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_quantize_reads_rows_apart_and_odd_addresses(b, dtype):
    base = torch.randn(70 * 400 + 3, generator=gen(5), device="cuda").to(TYPES[dtype])
    for offset, stride, cols in ((0, 400, 256), (1, 400, 256), (3, 257, 257), (0, 256, 130)):
        x = base[offset:].as_strided((70, cols), (stride, 1))
        check_quantized(*b.vptq_fp4_quantize(x), x)


def test_quantize_extremes(b):
    # zeros of both signs, the smallest subnormals, the largest values, every tie, and magnitudes on both sides of a scale's border
    x = torch.zeros(8, 256, device="cuda")
    x[0, ::2] = -0.0
    x[1, :32] = 1e-45
    x[1, 32:64] = -3.4028234e38
    x[1, 64:96] = 2.0 ** -126
    x[1, 96] = 1.5 * 2.0 ** -125
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], device="cuda")
    for i, s in enumerate((1.0, 2.0 ** -100, 2.0 ** 120)):
        x[2 + i, :8], x[2 + i, 32:40] = ties * s, -ties * s
    x[5, 0], x[5, 32], x[5, 64] = 7.0, 6.9999995, 3.5
    x[6, 0], x[6, 32], x[6, 64] = 3.4999998, 1.75, 1.7499999
    x[7, 0], x[7, 32] = 2.0 ** -127 * 7, 2.0 ** -127 * 3.4
    check_quantized(*b.vptq_fp4_quantize(x), x)
    for dtype in (torch.float16, torch.bfloat16):
        y = x.clamp(-6e4, 6e4).to(dtype)
        check_quantized(*b.vptq_fp4_quantize(y), y)


def test_quantize_every_fp16_value(b):
    x = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.float16)
    x = torch.where(x.isfinite(), x, torch.zeros_like(x))
    check_quantized(*b.vptq_fp4_quantize(x.view(512, 128)), x.view(512, 128))
    alone = torch.zeros(4096, 512, dtype=torch.float16, device="cuda")               # each value a block of its own
    alone.view(-1, 32)[:, 5] = x
    check_quantized(*b.vptq_fp4_quantize(alone), alone)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_quantize_shows_what_is_not_a_number(b, dtype, bad):
    x = torch.ones(3, 300, device="cuda", dtype=TYPES[dtype])
    x[1, 140] = bad
    x[2, 299] = bad
    q, s = b.vptq_fp4_quantize(x)
    check_quantized(q, s, x)
    for out in sorted(TYPES):
        v = b.vptq_fp4_values(q, s, 300, out)
        assert torch.isnan(v[1, 128:160]).all() and torch.isnan(v[2, 288:]).all() and torch.isfinite(v).sum() == 900 - 32 - 12


def test_quantize_no_rows(b):
    q, s = b.vptq_fp4_quantize(torch.zeros(0, 200, device="cuda", dtype=torch.float16))
    assert tuple(q.shape) == (0, 112) and tuple(s.shape) == (0, 2, 32, 16)
    assert tuple(b.vptq_fp4_values(q, s, 200).shape) == (0, 200)


# ---- values -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("out", sorted(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 32), (129, 1000), (300, 333), (2000, 776), (1, 4100)])
def test_values(b, rows, cols, out):
    q, s = ref.random_weight(rows, cols, gen(rows + cols), "cuda", 100, 140)
    want = ref.values(q, s, cols).to(TYPES[out])
    assert same(b.vptq_fp4_values(q, s, cols, out), want)
    given = torch.empty(rows, cols, dtype=TYPES[out], device="cuda")
    assert b.vptq_fp4_values(q, s, cols, out=given) is given and same(given, want)


def test_values_of_every_scale(b):
    q = torch.arange(256, device="cuda", dtype=torch.uint8).repeat(256, 1)             # every pair of codes in every row
    s = ref.scale_tiles(torch.arange(256, device="cuda", dtype=torch.uint8)[:, None].repeat(1, 16))
    got, want = b.vptq_fp4_values(q, s, 512, "fp32"), ref.values(q, s, 512).float()
    assert got[255].isnan().all() and same(got[:255], want[:255])
    got, want = b.vptq_fp4_values(q, s, 512, "bf16"), ref.values(q, s, 512).float().bfloat16()
    assert got[255].isnan().all() and same(got[:255], want[:255])


# ---- restore ----------------------------------------------------------------------------------------

SPECS = [synth.LayerSpec("q_rows", 300, 260, v=8, k1=256, k2=16), synth.LayerSpec("q_v12_out", 500, 390, v=12, k1=4096, n_out=130, v0=4, k0=16),
         synth.LayerSpec("q_v5", 129, 128, v=5, k1=37), synth.LayerSpec("q_v32", 257, 131, v=32, k1=40, n_out=3, v0=7, k0=9)]
# (large enough that the tables are staged in shared memory)
STAGED = [synth.LayerSpec("q_s8", 1000, 1100, v=8, k1=256), synth.LayerSpec("q_s8_res", 1003, 1101, v=8, k1=256, k2=256),
          synth.LayerSpec("q_s6_out", 1000, 1102, v=6, k1=256, k2=64, n_out=33, v0=4, k0=16),
          synth.LayerSpec("q_s6_12", 4100, 2006, v=6, k1=4096, n_out=130, v0=2, k0=64), synth.LayerSpec("q_s8_perm", 1000, 1100, v=8, k1=256, k2=16, permuted=True),
          synth.LayerSpec("q_l2_16", 500, 1030, v=8, k1=65536, k2=256, n_out=5, v0=8, k0=256), synth.LayerSpec("q_l2_groups", 500, 1024, v=8, k1=4096, n_groups=4)]


@pytest.mark.parametrize("spec", synth.small_specs() + SPECS, ids=lambda s: s.name)
def test_dequant_fp4_is_the_quantized_restored_weight(b, spec):
    d = synth.make_layer(spec, 0, 3, 1)
    check_quantized(*b.DeviceLayer(d).dequant_fp4(), torch.from_numpy(oracle.Layer.from_synth(d).dequant()).cuda())


# (a vector row of 128 columns to a warp: both tables staged or the residual's, with and without scale, outliers beside other columns, odd ends)
ROWS = [synth.LayerSpec("q_r8", 4100, 2006, v=8, k1=65536, k2=256, n_out=5, v0=8, k0=256), synth.LayerSpec("q_r6", 4001, 1030, v=6, k1=65536, k2=200, n_out=33, v0=4, k0=16),
        synth.LayerSpec("q_r8_plain", 2049, 1500, v=8, k1=2500, k2=200, has_scale=False), synth.LayerSpec("q_r6_wide", 1300, 4101, v=6, k1=4096, k2=256, n_out=130, v0=5, k0=100),
        synth.LayerSpec("q_r8_both", 3001, 1001, v=8, k1=256, k2=256, n_out=3, v0=8, k0=16), synth.LayerSpec("q_r6_both", 6000, 2100, v=6, k1=200, k2=150, n_out=33, v0=4, k0=16),
        synth.LayerSpec("q_r6_low", 7, 60001, v=6, k1=200, has_scale=False), synth.LayerSpec("q_r8_one", 1, 40000, v=8, k1=130)]


@pytest.mark.parametrize("spec", STAGED + ROWS, ids=lambda s: s.name)
def test_dequant_fp4_of_larger_layers(b, spec):
    dl = b.DeviceLayer(synth.make_layer(spec, 0, 3, 1))
    q, s = dl.dequant_fp4()
    check_quantized(q, s, dl.dequant())
    assert all(same(x, y) for x, y in zip(b.vptq_fp4_quantize(dl.dequant()), (q, s)))


def test_dequant_fp4_of_values_that_overflow(b):
    spec = synth.LayerSpec("q_inf", 130, 100, v=8, k1=16)
    d = synth.make_layer(spec, 0, 3, 1)
    d["c1"][:] = 60000
    d["scale"][:] = 1
    d["scale"][40] = 2
    dl = b.DeviceLayer(d)
    q, s = dl.dequant_fp4()
    check_quantized(q, s, dl.dequant())
    assert b.vptq_fp4_values(q, s, 100, "fp32")[:, 32:64].isnan().all()


# ---- product ----------------------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (8, 32, 1), (64, 64, 3), (65, 100, 7), (128, 256, 16), (200, 300, 17), (129, 31, 128), (1000, 2048, 77), (256, 224, 129), (4741, 208, 133),
          (520, 4104, 300), (4096, 4096, 1), (1024, 8192, 40), (2048, 1024, 255), (7, 5000, 5), (1500, 999, 600), (37888, 160, 100), (3000, 1100, 2), (448, 777, 8)]


@pytest.mark.parametrize("x_type", ["fp16", "bf16", "e2m1"])
@pytest.mark.parametrize("M,N,B", SHAPES)
def test_linear(b, M, N, B, x_type):
    g = gen(M + 3 * N + 7 * B)
    w, ws = ref.random_weight(M, N, g, "cuda")
    x = torch.randn(B, N, generator=g, device="cuda") * torch.exp(2 * torch.randn(B, 1, generator=g, device="cuda"))
    for out in sorted(TYPES):
        if x_type == "e2m1":
            q, s = ref.random_weight(B, N, g, "cuda")
            check_linear(b, q, w, ws, out, N, ref.values(q, s, N), s)
        else:
            v = x.to(TYPES[x_type])
            y = check_linear(b, v, w, ws, out, N, ref.quantize(v)[0])
            q, s = b.vptq_fp4_quantize(v)
            assert same(y, b.vptq_linear_fp4(q, w, ws, x_scale=s, out_dtype=out))


# (every form of the tensor-core kernel: pairs and single CTAs of each width, splits over clusters)
@pytest.mark.parametrize("M,N,B", [(8192, 512, 2048), (6144, 512, 1000), (4096, 300, 1100), (14336, 520, 500), (28672, 256, 300), (9472, 1024, 16), (18944, 512, 16),
                                   (128, 8192, 16), (300, 8192, 200), (2000, 16384, 30), (10000, 288, 128), (28416, 290, 120), (4096, 8192, 300), (2000, 4096, 129), (1000, 2048, 500), (3000, 1100, 400), (520, 16384, 1000),
                                   (1001, 4200, 257)])
def test_linear_of_many_shapes(b, M, N, B):
    g = gen(M + N + B)
    w, ws = ref.random_weight(M, N, g, "cuda")
    q, s = ref.random_weight(B, N, g, "cuda")
    y = check_linear(b, q, w, ws, "fp32", N, ref.values(q, s, N), s)
    assert same(y, b.vptq_linear_fp4(q, w, ws, x_scale=s, out_dtype="fp32"))            # bit for bit the same every time


# (few tokens: warps with and without columns, rows that begin and end inside a tile of scales, one group or two a CTA; and those that the other kernel takes)
@pytest.mark.parametrize("B", [1, 2, 7, 8, 9, 15, 16])
@pytest.mark.parametrize("M,N", [(1, 64), (32, 8192), (33, 2560), (100, 5000), (1024, 1000), (1001, 4096), (4100, 1100), (4736, 300), (9000, 640), (28672, 512), (37888, 260),
                                 (40001, 130), (80000, 256), (300, 40000), (5000, 17000)])
def test_linear_of_few_tokens(b, M, N, B):
    g = gen(M + N + B)
    w, ws = ref.random_weight(M, N, g, "cuda")
    q, s = ref.random_weight(B, N, g, "cuda")
    y = check_linear(b, q, w, ws, "fp32", N, ref.values(q, s, N), s)
    assert same(y, b.vptq_linear_fp4(q, w, ws, x_scale=s, out_dtype="fp32"))
    x = torch.randn(B, N, generator=g, device="cuda").half()
    check_linear(b, x, w, ws, "bf16", N, ref.quantize(x)[0])


def test_linear_paths(b):
    path = lambda M, N, B, x="fp16": (b.vptq_linear_fp4_path(b.make_fp4_desc(M, N, x), B), b.vptq_linear_fp4_launches(b.make_fp4_desc(M, N, x), B))  # noqa: E731
    few, two, one = ("fp4_few", 1), ("fp4_tcgen05", 2), ("fp4_tcgen05", 1)
    assert [path(4096, 4096, B) for B in (1, 8, 9, 300)] == [few, few, two, two] and [path(4096, 4096, B, "e2m1") for B in (1, 300)] == [one, one]
    assert [path(M, N, 1, "bf16") for M, N in ((4096, 4104), (40960, 64), (64, 100))] == [two] * 3


def test_linear_of_every_scale(b):
    """The rows' and the weight's scales run over all bytes, with sums that neither overflow nor lose to FP32's smallest values; 255 reads as NaN."""
    g = gen(9)
    M, N, B = 256, 512, 256
    w, _ = ref.random_weight(M, N, g, "cuda")
    q, _ = ref.random_weight(B, N, g, "cuda")
    for middle in (70, 127, 180):
        bytes_ = torch.randint(middle - 3, middle + 4, (M, 16), generator=g, device="cuda", dtype=torch.uint8)
        ws, s = ref.scale_tiles(bytes_), ref.scale_tiles(254 - bytes_)
        check_linear(b, q, w, ws, "fp32", N, ref.values(q, s, N), s)
    # powers below FP32's normal range, and near its end, of the weight and of the tokens
    bytes_ = torch.randint(120, 130, (M, 16), generator=g, device="cuda", dtype=torch.uint8)
    ends = bytes_.clone()
    ends[7], ends[8], ends[9, ::2] = 0, 235, 0
    y = check_linear(b, q, w, ref.scale_tiles(ends), "fp32", N, ref.values(q, ref.scale_tiles(bytes_), N), ref.scale_tiles(bytes_))
    assert y[:, 7].any()
    check_linear(b, q, w, ref.scale_tiles(bytes_), "fp32", N, ref.values(q, ref.scale_tiles(ends), N), ref.scale_tiles(ends))
    bytes_ = torch.full((M, 16), 127, device="cuda", dtype=torch.uint8)
    one = ref.scale_tiles(bytes_)
    bytes_ = bytes_.clone()
    bytes_[5, 3] = bytes_[200, 15] = 255
    bad = ref.scale_tiles(bytes_)
    clean = b.vptq_linear_fp4(q, w, one, x_scale=one, out_dtype="fp32")
    y = b.vptq_linear_fp4(q, w, bad, x_scale=one, out_dtype="fp32")
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[5] = keep[200] = False
    assert y[:, ~keep].isnan().all() and same(y[:, keep], clean[:, keep])
    y = b.vptq_linear_fp4(q, w, one, x_scale=bad, out_dtype="fp32")
    assert y[~keep].isnan().all() and same(y[keep], clean[keep])


@pytest.mark.parametrize("B", [1, 5])
def test_linear_of_few_tokens_and_every_scale(b, B):
    g = gen(B)
    M, N = 300, 512
    w, _ = ref.random_weight(M, N, g, "cuda")
    bytes_ = torch.randint(100, 140, (M, 16), generator=g, device="cuda", dtype=torch.uint8)
    bytes_[7], bytes_[8] = 0, 250                                      # powers below FP32's normal range, and near its end
    w[8] &= 0x33
    x = torch.randn(B, N, generator=g, device="cuda").bfloat16()
    ws = ref.scale_tiles(bytes_)
    clean = check_linear(b, x, w, ws, "fp32", N, ref.quantize(x)[0])
    assert clean[:, 7].any() and b.vptq_linear_fp4_path(b.make_fp4_desc(M, N, "bf16"), B) == "fp4_few"
    bytes_[5, 3] = bytes_[299, 15] = 255
    w[299] = 0                                                         # zeros times what is no number
    y = b.vptq_linear_fp4(x, w, ref.scale_tiles(bytes_), out_dtype="fp32")
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[5] = keep[299] = False
    assert y[:, ~keep].isnan().all() and same(y[:, keep], clean[:, keep])


@pytest.mark.parametrize("B", [1, 5, 8, 40, 300])
@pytest.mark.parametrize("size", [-126, -119, -110, -30, 0, 100, 116, 118, 124])
def test_linear_of_scales_that_cancel(b, size, B):
    """Weight and tokens near opposite ends of FP32's range: the results are in the middle of it."""
    g = gen(B + size)
    M, N = 300, 512
    bytes_ = torch.randint(max(0, 119 - size), min(254, 127 - size) + 1, (M, 16), generator=g, device="cuda", dtype=torch.uint8)
    w, _ = ref.random_weight(M, N, g, "cuda")
    x = (torch.randn(B, N, generator=g, device="cuda").clamp(-3, 3) * 2.0 ** size).bfloat16()
    ws = ref.scale_tiles(bytes_)
    y = check_linear(b, x, w, ws, "fp32", N, ref.quantize(x)[0])
    q, s = b.vptq_fp4_quantize(x)
    check_linear(b, q, w, ws, "fp32", N, ref.values(q, s, N), s)
    assert y.isfinite().all() and y.any()


@pytest.mark.parametrize("B", [1, 40, 300])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_linear_keeps_what_is_not_a_number_in_its_row(b, B, bad):
    g = gen(B)
    w, ws = ref.random_weight(500, 700, g, "cuda")
    x = torch.randn(B, 700, generator=g, device="cuda").half()
    clean = b.vptq_linear_fp4(x, w, ws)
    row = B // 2
    x[row, 333] = bad
    y = b.vptq_linear_fp4(x, w, ws)
    keep = torch.arange(B, device="cuda") != row
    assert y[row].isnan().all() and same(y[keep], clean[keep])


def test_linear_rows_and_columns_of_zeros(b):
    g = gen(1)
    w, ws = ref.random_weight(300, 512, g, "cuda")
    x = torch.zeros(20, 512, device="cuda", dtype=torch.bfloat16)
    assert not b.vptq_linear_fp4(x, w, ws).any()
    x[3] = 1.0
    y = b.vptq_linear_fp4(x, w, ws, out_dtype="fp32")
    assert y[3].any() and not y[:3].any() and not y[4:].any()


def test_a_restored_layer_runs_through_the_product(b):
    """Restore, product of a prompt and of one token, and the fully quantized chain of two layers, against 64 bits."""
    d1, d2 = (synth.make_layer(synth.LayerSpec(f"q_chain{i}", M, N, v=8, k1=256, k2=256), 0, i, 1) for i, (M, N) in enumerate(((1000, 512), (512, 1000))))
    l1, l2 = b.DeviceLayer(d1), b.DeviceLayer(d2)
    (w1, s1), (w2, s2) = l1.dequant_fp4(), l2.dequant_fp4()
    for B in (1, 50):
        x = torch.randn(B, 512, generator=gen(B), device="cuda").half()
        h = check_linear(b, x, w1, s1, "bf16", 512, ref.quantize(x)[0])
        check_linear(b, h, w2, s2, "fp32", 1000, ref.quantize(h)[0])
        # A code is off by at most a fifth of a value of at least its scale, and by at most a quarter of the scale below.  Evenly spread over
        # that, x's and the weight's errors are each less than 0.25 / sqrt(3) of the values, and independent: at most 0.21 together.
        exact = x.double() @ l1.dequant().double().t()
        assert float((h.double() - exact).norm() / exact.norm()) < 0.25
