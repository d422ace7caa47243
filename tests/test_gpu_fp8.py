"""8-bit floating point operators against their definitions in 64 bits."""
import pytest
import torch

import fp8_reference as ref
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


def check_quantized(q, scale, x, block_rows):
    rows, cols = x.shape
    want, want_scale = ref.quantize(x, block_rows)
    assert q.dtype == torch.float8_e4m3fn and tuple(q.shape) == (rows, ref.pitch(cols))
    assert torch.equal(scale, want_scale)
    # (FP16 inputs of the widest rows overflow: a value of an infinite block is a NaN on both sides)
    got = q[:, :cols].double()
    assert ((got == want) | (got.isnan() & want.isnan())).all()
    assert not q[:, cols:].view(torch.uint8).any()                      # pad bytes are zeros


# ---- quantization -----------------------------------------------------------------------------------

@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (2, 15), (3, 128), (127, 129), (128, 16), (129, 1000), (300, 333), (1, 7), (2000, 776)])
def test_quantize(b, rows, cols, dtype, block_rows):
    g = gen(rows * 1000 + cols)
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(3 * torch.randn(rows, 1, generator=g, device="cuda"))
    x = x.to(TYPES[dtype])
    check_quantized(*b.vptq_fp8_quantize(x, block_rows), x, block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_quantize_reads_rows_apart_and_odd_addresses(b, dtype, block_rows):
    g = gen(5)
    base = torch.randn(70 * 400 + 3, generator=g, device="cuda").to(TYPES[dtype])
    for offset, stride, cols in ((0, 400, 256), (1, 400, 256), (3, 257, 257), (0, 256, 130)):
        x = base[offset:].as_strided((70, cols), (stride, 1))
        check_quantized(*b.vptq_fp8_quantize(x, block_rows), x, block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_extremes(b, block_rows):
    # zeros, the smallest subnormals, the largest values, ties of e4m3 (the block's maximum 448 makes scale and factor 1)
    x = torch.zeros(4, 512, device="cuda")
    x[0, :128] = 1e-45
    x[0, 128:256] = 3.4e38
    x[0, 256] = 448
    x[0, 257:257 + 14] = torch.tensor([1.0625, 1.1875, -1.0625, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 0.0, -0.0, 440.0, 432.0, 2.0 ** -11, 464.0 / 2, 1e-30],
                                      device="cuda")
    check_quantized(*b.vptq_fp8_quantize(x, block_rows), x, block_rows)
    for dtype in (torch.float16, torch.bfloat16):
        check_quantized(*b.vptq_fp8_quantize(x.clamp(-6e4, 6e4).to(dtype), block_rows), x.clamp(-6e4, 6e4).to(dtype), block_rows)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_quantize_shows_what_is_not_a_number(b, dtype, bad):
    x = torch.ones(3, 300, device="cuda", dtype=TYPES[dtype])
    x[1, 140] = bad
    q, s = b.vptq_fp8_quantize(x)
    v = ref.values(q, s, 300, 1)
    assert torch.isnan(v[1, 128:256]).all() and torch.isfinite(v[1, :128]).all() and torch.isfinite(v[1, 256:]).all()
    assert torch.isfinite(v[0]).all() and torch.isfinite(v[2]).all() and not q[:, 300:].view(torch.uint8).any()
    q, s = b.vptq_fp8_quantize(x, 128)
    v = ref.values(q, s, 300, 128)
    assert torch.isnan(v[:, 128:256]).all() and torch.isfinite(v[:, :128]).all() and not q[:, 300:].view(torch.uint8).any()


def test_quantize_no_rows(b):
    q, s = b.vptq_fp8_quantize(torch.zeros(0, 200, device="cuda", dtype=torch.float16))
    assert tuple(q.shape) == (0, 208) and tuple(s.shape) == (0, 2)


# ---- restore ----------------------------------------------------------------------------------------

MORE = [synth.LayerSpec("f_rows", 300, 260, v=8, k1=256, k2=16), synth.LayerSpec("f_v12_out", 500, 390, v=12, k1=4096, n_out=130, v0=4, k0=16),
        synth.LayerSpec("f_v5", 129, 128, v=5, k1=37), synth.LayerSpec("f_v32", 257, 131, v=32, k1=40, n_out=3, v0=7, k0=9)]


@pytest.mark.parametrize("spec", synth.small_specs() + MORE, ids=lambda s: s.name)
def test_dequant_fp8_is_the_quantized_restored_weight(b, spec):
    d = synth.make_layer(spec, 0, 3, 1)
    q, scale = b.DeviceLayer(d).dequant_fp8()
    W = torch.from_numpy(oracle.Layer.from_synth(d).dequant()).cuda()
    check_quantized(q, scale, W, 128)


# (large enough that the tables are staged in shared memory; index widths of 8, 12 and 16 bits and others, columns that start and end
# inside a block, rows that cross its edge)
STAGED = [synth.LayerSpec("f_s8", 1000, 1100, v=8, k1=256), synth.LayerSpec("f_s8_res", 1003, 1101, v=8, k1=256, k2=256), synth.LayerSpec("f_s6_out", 1000, 1102, v=6, k1=256, k2=64, n_out=33, v0=4, k0=16),
          synth.LayerSpec("f_s6_12", 4100, 2006, v=6, k1=4096, n_out=130, v0=2, k0=64), synth.LayerSpec("f_s8_perm", 1000, 1100, v=8, k1=256, k2=16, permuted=True),
          synth.LayerSpec("f_l2_16", 500, 1030, v=8, k1=65536, k2=256, n_out=5, v0=8, k0=256), synth.LayerSpec("f_l2_groups", 500, 1024, v=8, k1=4096, n_groups=4)]


@pytest.mark.parametrize("spec", STAGED, ids=lambda s: s.name)
def test_dequant_fp8_of_larger_layers(b, spec):
    dl = b.DeviceLayer(synth.make_layer(spec, 0, 3, 1))
    check_quantized(*dl.dequant_fp8(), dl.dequant(), 128)


def test_dequant_fp8_scale_per_row(b):
    spec = synth.LayerSpec("f_scale_rows", 200, 200, v=8, k1=256, n_out=5, v0=4, k0=16)
    d = synth.make_layer(spec, 0, 3, 1)
    dl = b.DeviceLayer(d, scale_rows=True)
    check_quantized(*dl.dequant_fp8(), dl.dequant(), 128)


def test_dequant_fp8_survives_a_list_that_is_no_permutation(b):
    spec = synth.LayerSpec("f_bad_perm", 130, 200, v=8, k1=256, permuted=True)
    d = synth.make_layer(spec, 0, 3, 1)
    d["col_perm"][:] = 7
    d["col_perm"][5] = -3
    dl = b.DeviceLayer(d)
    q, scale = dl.dequant_fp8()
    v = ref.values(q, scale, 200, 128)
    assert torch.isfinite(v).all()
    assert v[:, 7].any() and v[:, 199].any()                            # the entry outside [0, N) counts as N - 1
    v[:, 7] = 0
    v[:, 199] = 0
    assert not v.any()                                                  # no stored column names the other features


# ---- the product ------------------------------------------------------------------------------------

def operands(M, N, B, x_type, seed):
    g = gen(seed)
    w, ws = ref.random_weight(M, N, g, "cuda")
    x = torch.randn(B, N, generator=g, device="cuda") * (1 + 20 * (torch.rand(N, generator=g, device="cuda") < 0.02))
    if x_type == "e4m3":
        q = torch.zeros(B, ref.pitch(N), dtype=torch.float8_e4m3fn, device="cuda")
        q[:, :N] = (x * 30).clamp(-448, 448).to(torch.float8_e4m3fn)
        xs = torch.rand(B, -(-N // 128), generator=g, device="cuda") + 0.1
        return w, ws, q, xs, ref.values(q, xs, N, 1)
    x = x.to(TYPES[x_type])
    v, s = ref.quantize(x, 1)
    return w, ws, x, None, v * ref.expand(s, B, N, 1)


def check_linear(b, M, N, B, x_type, out, seed=1):
    w, ws, x, xs, xv = operands(M, N, B, x_type, seed)
    y = b.vptq_linear_fp8(x, w, ws, x_scale=xs, out_dtype=out)
    want, bound = ref.linear(xv, ref.values(w, ws, N, 128), TYPES[out], -(-N // 128))
    assert y.dtype == TYPES[out] and tuple(y.shape) == (B, M)
    off = (y.double() - want).abs()
    assert (off <= bound).all(), float((off / bound).max())
    return y


@pytest.mark.parametrize("x_type", ["e4m3", "fp16", "bf16"])
@pytest.mark.parametrize("M,N,B", [(1, 1, 1), (1, 128, 3), (16, 16, 1), (15, 100, 8), (17, 129, 9), (130, 1030, 16), (300, 128, 7), (128, 2048, 2),
                                   (513, 1000, 1), (64, 4104, 5), (260, 333, 15), (1000, 640, 4)])
def test_linear_few_tokens(b, M, N, B, x_type):
    if x_type == "e4m3":
        N = ref.pitch(N)                            # e4m3 rows have no other width
    check_linear(b, M, N, B, x_type, "fp32")


@pytest.mark.parametrize("x_type", ["e4m3", "fp16", "bf16"])
@pytest.mark.parametrize("M,N,B", [(1, 16, 17), (130, 144, 33), (64, 1040, 100), (257, 512, 128), (384, 400, 129), (1000, 2064, 300), (260, 333, 40)])
def test_linear_many_tokens(b, M, N, B, x_type):
    if x_type == "e4m3":
        N = ref.pitch(N)
    check_linear(b, M, N, B, x_type, "fp32")


# (tiles of every width, alone and in pairs, and tiles split over 2, 4 and 8 CTAs; rows of the result that are no multiple of 16 bytes)
@pytest.mark.parametrize("M,N,B,out", [(128, 4096, 40, "fp32"), (1000, 2048, 77, "fp16"), (2048, 1024, 128, "bf16"), (4096, 1024, 64, "fp16"), (4099, 512, 100, "fp32"),
                                       (9472, 256, 128, "fp16"), (18944, 272, 100, "bf16"), (37888, 160, 17, "fp16"), (33152, 128, 33, "bf16"), (9472, 400, 512, "fp16"),
                                       (18944, 144, 300, "fp32"), (14208, 256, 512, "bf16"), (16576, 384, 513, "fp16"), (28416, 128, 385, "fp32"), (1001, 1000, 1111, "bf16"), (18990, 128, 40, "fp16"),
                                       (4744, 128, 133, "bf16"), (4741, 200, 133, "fp32"), (9760, 128, 150, "fp16"), (15120, 144, 200, "fp32"), (15121, 128, 129, "bf16")])
def test_linear_tiles(b, M, N, B, out):
    N = ref.pitch(N)
    check_linear(b, M, N, B, "e4m3", out)


@pytest.mark.parametrize("B", [17, 100, 600])
def test_linear_reports_no_error(b, B):
    w, ws, x, _, _ = operands(500, 640, B, "fp16", 3)
    desc = b.make_fp8_desc(500, 640, "fp16", "fp16")
    room = torch.full((b.vptq_linear_fp8_workspace_bytes(desc, B),), 255, dtype=torch.uint8, device="cuda")       # what it held before does not matter
    y = b.vptq_linear_fp8(x, w, ws, workspace=room)
    assert b.vptq_linear_fp8_path(desc, B) == "fp8_tcgen05" and b.vptq_workspace_status(room) == b.OK
    assert same(y, b.vptq_linear_fp8(x, w, ws))


@pytest.mark.parametrize("out", ["fp16", "bf16"])
@pytest.mark.parametrize("M,N,B", [(130, 1030, 5), (256, 512, 16), (300, 1000, 48), (264, 768, 200)])
def test_linear_result_types(b, M, N, B, out):
    check_linear(b, M, N, B, "bf16", out)


@pytest.mark.parametrize("B", [1, 8, 16, 17, 130])
@pytest.mark.parametrize("N", [1024, 1000, 333])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_quantizing_inside_the_call_gives_the_same_bits(b, B, N, dtype):
    w, ws, x, _, _ = operands(390, N, B, dtype, 4)
    q, s = b.vptq_fp8_quantize(x)
    a = b.vptq_linear_fp8(x, w, ws, out_dtype="fp32")
    assert same(a, b.vptq_linear_fp8(q, w, ws, x_scale=s, out_dtype="fp32"))
    assert same(a, b.vptq_linear_fp8(x, w, ws, out_dtype="fp32"))                    # and again


@pytest.mark.parametrize("B", [3, 40])
def test_not_a_number_stays_in_its_token(b, B):
    w, ws, x, _, _ = operands(200, 512, B, "fp16", 6)
    clean = b.vptq_linear_fp8(x, w, ws, out_dtype="fp32")
    x[1, 200] = float("nan")
    x[2, 300] = float("inf")
    y = b.vptq_linear_fp8(x, w, ws, out_dtype="fp32")
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
    rest = [t for t in range(B) if t not in (1, 2)]
    assert same(y[rest], clean[rest])


@pytest.mark.parametrize("B", [4, 50])
def test_linear_of_zeros_and_of_tiny_values(b, B):
    w, ws, x, _, _ = operands(100, 300, B, "bf16", 7)
    x.zero_()
    assert not b.vptq_linear_fp8(x, w, ws, out_dtype="fp32").any()
    x.fill_(1e-38)                                   # far below 2^-100 / 448: rounds to zero
    assert not b.vptq_linear_fp8(x, w, ws, out_dtype="fp32").any()


@pytest.mark.parametrize("B", [2, 16, 64, 200])
def test_linear_writes_its_result_and_nothing_else(b, B):
    M = 200
    w, ws, x, _, _ = operands(M, 384, B, "fp16", 8)
    room = torch.full(((B + 2) * M,), 77.0, dtype=torch.float16, device="cuda")
    out = room[M:-M].view(B, M)
    y = b.vptq_linear_fp8(x, w, ws, out=out)
    assert y is out and (room[:M] == 77).all() and (room[-M:] == 77).all()
    assert same(out, b.vptq_linear_fp8(x, w, ws, out_dtype="fp16"))


@pytest.mark.parametrize("B", [1, 16, 70, 300])
def test_other_streams_and_replayed_graphs(b, B):
    w, ws, x, _, _ = operands(520, 1000, B, "fp16", 9)
    want = b.vptq_linear_fp8(x, w, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = b.vptq_linear_fp8(x, w, ws)
    side.synchronize()
    assert same(y, want)
    graph, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, s = b.vptq_fp8_quantize(x)
        a = b.vptq_linear_fp8(q, w, ws, x_scale=s, out_dtype="fp16")
        c = b.vptq_linear_fp8(x, w, ws)
    with torch.cuda.graph(two):
        e = b.vptq_linear_fp8(x, w, ws)
    x.mul_(0.5)
    want = b.vptq_linear_fp8(x, w, ws)
    for _ in range(3):
        a.zero_(), c.zero_(), e.zero_()
        graph.replay()
        two.replay()
        torch.cuda.synchronize()
        assert same(a, want) and same(c, want) and same(e, want)


@pytest.mark.parametrize("B", [1, 8, 16, 300])
def test_weights_written_just_before(b, B):
    M, N = 1100, 1024
    g = gen(10)
    x = torch.randn(B, N, generator=g, device="cuda").half()
    Ws = [(torch.randn(M, N, generator=g, device="cuda") * (i + 1)).half() for i in range(6)]
    want = []
    for W in Ws:
        q, s = b.vptq_fp8_quantize(W, 128)
        torch.cuda.synchronize()
        want.append(b.vptq_linear_fp8(x, q, s, out_dtype="fp32"))
        torch.cuda.synchronize()
    def all_of_them():
        got, q, s = [], None, None
        for W in Ws:
            del q, s                                 # the next ones take their place
            q, s = b.vptq_fp8_quantize(W, 128)
            got.append(b.vptq_linear_fp8(x, q, s, out_dtype="fp32"))
        return got
    assert all(same(a, w) for a, w in zip(all_of_them(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of_them()
    for _ in range(3):
        for a in got:
            a.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(a, w) for a, w in zip(got, want))


def test_one_row_of_activations_as_a_weight(b):
    # one row's scales have the same shape either way: what the quantizer has just written may be the weight
    g = gen(11)
    x = torch.randn(4, 4096, generator=g, device="cuda").half()
    rows = [torch.randn(1, 4096, generator=g, device="cuda").half() for _ in range(4)]
    want = []
    for r in rows:
        q, s = b.vptq_fp8_quantize(r)
        torch.cuda.synchronize()
        want.append(b.vptq_linear_fp8(x, q, s))
        torch.cuda.synchronize()
    q = s = None
    for r, w in zip(rows, want):
        del q, s
        q, s = b.vptq_fp8_quantize(r)
        assert same(b.vptq_linear_fp8(x, q, s), w)


@pytest.mark.parametrize("B", [2, 16, 77, 300])
def test_two_calls_at_once(b, B):
    w, ws, x, _, _ = operands(4096, 4096, B, "bf16", 12)
    other = (x * 0.5).contiguous()
    want, want_other = b.vptq_linear_fp8(x, w, ws), b.vptq_linear_fp8(other, w, ws)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i, t in enumerate((x, other)):
            with torch.cuda.stream(streams[i]):
                got[i].append(b.vptq_linear_fp8(t, w, ws))
    torch.cuda.synchronize()
    assert all(same(y, want) for y in got[0]) and all(same(y, want_other) for y in got[1])


def test_a_layer_restored_once_runs_its_prompts(b):
    """The operators together, as a program uses them: a vector-quantized layer, restored to e4m3, takes a prompt; single tokens stay
    on the compressed layer."""
    spec = synth.LayerSpec("f_together", 520, 1030, v=8, k1=65536, k2=256, x_dtype="bf16", out_dtype="fp32")
    d = synth.make_layer(spec, 0, 3, 70)
    dl = b.DeviceLayer(d)
    q, scale = dl.dequant_fp8()
    x = dl.upload_x(d["x"])
    y = b.vptq_linear_fp8(x, q, scale, out_dtype="fp32")
    W = torch.from_numpy(oracle.Layer.from_synth(d).dequant()).cuda()
    wv, wsc = ref.quantize(W, 128)
    xv, xsc = ref.quantize(x, 1)
    want, bound = ref.linear(xv * ref.expand(xsc, 70, 1030, 1), wv * ref.expand(wsc, 520, 1030, 128), torch.float32, 9)
    assert ((y.double() - want).abs() <= bound).all()
    # against the layer itself: two roundings of half an e4m3 step, 2^-4 each, of every product, at random signs: the sum of 1030
    # products is off by about 2^-4 * sqrt(2 / 3) of its root mean square (uniform in half a step); 2^-4 has room for it
    full = dl.linear(x).double()
    assert float((y.double() - full).norm() / full.norm()) < 2.0 ** -4
