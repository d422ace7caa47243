"""Calls of the 4-bit floating point operators that a program makes beside the plain ones: parts of stacked operands, empty batches, workspaces,
other streams, calls that overlap, replayed graphs, and device-side waits that run out."""
import pytest
import torch

import fp4_reference as ref
from paper_2409_17066_b200 import synth
from test_gpu_fp4 import same
from test_gpu_fp8_waits import right_or_nan, with_short_waits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_parts_of_stacks(b):
    g = gen(1)
    both = [ref.random_weight(200, 390, g, "cuda") for _ in range(3)]
    w, s = (torch.stack([t[i] for t in both]) for i in range(2))
    x = torch.randn(30, 390, generator=g, device="cuda").half()
    for e in range(3):
        assert same(b.vptq_linear_fp4(x, w[e], s[e]), b.vptq_linear_fp4(x, *both[e]))
        assert same(b.vptq_fp4_values(w[e], s[e], 390), b.vptq_fp4_values(*both[e], 390))
    # rows of the weight from a tile of scales on
    assert same(b.vptq_linear_fp4(x, w[0][128:], s[0][1:]), b.vptq_linear_fp4(x, w[0], s[0])[:, 128:])


@pytest.mark.parametrize("N", [390, 391, 256])
@pytest.mark.parametrize("B", [1, 3, 40])
def test_some_tokens_of_a_batch(b, B, N):
    """Activations that start at any value."""
    g = gen(N)
    w, s = ref.random_weight(130, N, g, "cuda")
    x = torch.randn(B + 3, N, generator=g, device="cuda").bfloat16()
    for t in range(4):
        assert same(b.vptq_linear_fp4(x[t:t + B], w, s, out_dtype="fp32"), b.vptq_linear_fp4(x[t:t + B].clone(), w, s, out_dtype="fp32"))


@pytest.mark.parametrize("x_type", ["fp16", "bf16", "e2m1"])
def test_an_empty_batch(b, x_type):
    w, s = ref.random_weight(130, 256, gen(4), "cuda")
    x, xs = torch.empty(0, 256, device="cuda", dtype=torch.bfloat16 if x_type == "bf16" else torch.float16), None
    if x_type == "e2m1":
        x, xs = b.vptq_fp4_quantize(x)
    y = b.vptq_linear_fp4(x, w, s, x_scale=xs)
    assert tuple(y.shape) == (0, 130) and y.dtype == (torch.float16 if x_type == "fp16" else torch.bfloat16)
    out = torch.empty(0, 130, device="cuda")
    assert b.vptq_linear_fp4(x, w, s, x_scale=xs, out=out) is out
    with pytest.raises(AssertionError):
        b.vptq_linear_fp4(x, w, s, x_scale=xs, out=torch.empty(0, 131, device="cuda"))


def test_refusals(b):
    g = gen(5)
    w, s = ref.random_weight(130, 256, g, "cuda")
    x = torch.randn(20, 256, generator=g, device="cuda").half()
    q, qs = b.vptq_fp4_quantize(x)
    with pytest.raises(b.VptqError):
        b.vptq_linear_fp4(x.float(), w, s)
    spread = torch.zeros(1 << 21, 2, dtype=torch.uint8, device="cuda")[:, 0]
    for bad in (lambda: b.vptq_linear_fp4(x, w, s, x_scale=qs), lambda: b.vptq_linear_fp4(q, w, s), lambda: b.vptq_linear_fp4(x[:, :255], w, s), lambda: b.vptq_linear_fp4(x[:, :128].contiguous(), w, s),
                lambda: b.vptq_linear_fp4(x, w, s[:1]), lambda: b.vptq_linear_fp4(x, w, s.view(2, 2, 512)), lambda: b.vptq_linear_fp4(q, w, s, x_scale=qs[:, :1]),
                lambda: b.vptq_linear_fp4(x, w, s, out=torch.empty(20, 130, device="cuda"), out_dtype="fp16"), lambda: b.vptq_linear_fp4(x, w, s, out=torch.empty(20, 131, device="cuda")),
                lambda: b.vptq_linear_fp4(x, w, s, workspace=spread), lambda: b.vptq_linear_fp4(x, w, s, workspace=torch.zeros(1 << 22, dtype=torch.uint8)),
                lambda: b.vptq_fp4_quantize(x[0]), lambda: b.vptq_fp4_quantize(x.t()), lambda: b.vptq_fp4_values(q, qs, 255 - 32), lambda: b.vptq_fp4_values(q, s, 256),
                lambda: b.vptq_fp4_values(q, qs, 256, out=torch.empty(20, 255, device="cuda")), lambda: b.vptq_fp4_values(q[::2], qs, 256)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(b.VptqError):
        b.vptq_linear_fp4(x, w, s, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(b.VptqError):
        b.vptq_fp4_values(q, qs, 0)
    assert not spread.any()


def test_refusals_of_the_cache(b):
    cache = b.make_cache(4, 8, 2, 64, "e2m1")
    i = torch.zeros(8, dtype=torch.int32, device="cuda")
    table, start, cu = i[:3].view(1, 3), i[:1], i[:2]
    k = torch.zeros(5, 2, 64, device="cuda")
    other = b.make_cache(4, 8, 2, 64, "e4m3")
    for bad in (lambda: b.vptq_cache_write(k[:, :1], k[:, :1], *cache, table, start, cu), lambda: b.vptq_cache_write(k, k[:4], *cache, table, start, cu),
                lambda: b.vptq_cache_write(k, k.half(), *cache, table, start, cu), lambda: b.vptq_cache_write(k.transpose(1, 2), k.transpose(1, 2), *cache, table, start, cu),
                lambda: b.vptq_cache_write(k[..., :60], k[..., :60], cache[0][..., :16], *cache[1:], table, start, cu), lambda: b.vptq_cache_write(k, k, *cache[:2], *other[2:], table, start, cu),
                lambda: b.vptq_cache_write(k, k, *cache, table.long(), start, cu), lambda: b.vptq_cache_write(k, k, *cache, table, i[:2], cu), lambda: b.vptq_cache_write(k, k, *cache, table, start, i[:3]),
                lambda: b.vptq_cache_write(k, k, *cache, table, start, cu.cpu()), lambda: b.vptq_cache_read(*cache, table, start, cu, 5, 65), lambda: b.vptq_cache_read(*cache, table, start, cu, 5, 64, k=k[:4]),
                lambda: b.vptq_cache_read(*cache, table, start, cu, 5, 64, "fp16", k=k), lambda: b.vptq_cache_read(*cache, table, start, cu, 5, 64, k=k, v=k.half())):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: b.vptq_cache_read(*cache, table, start, cu, -1, 64), lambda: b.vptq_cache_read(*cache, table, start, cu, 5, 0),
                lambda: b.vptq_cache_write(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn), *cache, table, start, cu)):
        with pytest.raises(b.VptqError):
            bad()
    assert not any(t.any() for t in cache)


def test_calls_on_two_streams_at_once(b):
    g = gen(6)
    w, s = ref.random_weight(4096, 2048, g, "cuda")
    xs = [torch.randn(B, 2048, generator=g, device="cuda").half() for B in (1, 16, 200)]
    want = [b.vptq_linear_fp4(x, w, s) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[] for _ in xs]
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(b.vptq_linear_fp4(xs[i], w, s))
    torch.cuda.synchronize()
    assert all(same(y, want[i]) for i in range(len(xs)) for y in got[i])


@pytest.mark.parametrize("B", [1, 12, 40, 300])
def test_products_in_a_replayed_graph(b, B):
    """Activations and weight change between the replays; two products one behind the other, the second over the first's results."""
    g = gen(7)
    (w, s), (w2, s2) = ref.random_weight(1000, 768, g, "cuda"), ref.random_weight(768, 1000, g, "cuda")
    x = torch.randn(B, 768, generator=g, device="cuda").half()
    chain = lambda: b.vptq_linear_fp4(b.vptq_linear_fp4(x, w, s), w2, s2, out_dtype="fp32")  # noqa: E731
    chain()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = chain()
    for i in range(3):
        x.copy_(torch.randn(B, 768, generator=g, device="cuda"))
        w.copy_(ref.random_weight(1000, 768, g, "cuda")[0])
        want = chain()
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(y, want)


@pytest.mark.parametrize("k2,permuted", [(16, False), (16, True), (0, False)])
def test_a_restore_in_a_replayed_graph(b, k2, permuted):
    dl = b.DeviceLayer(synth.make_layer(synth.LayerSpec("q_graph", 1000, 1100, v=8, k1=256, k2=k2, permuted=permuted), 0, 3, 1))
    dl.dequant_fp4()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, s = dl.dequant_fp4()
        v = b.vptq_fp4_values(q, s, 1100)
    dl.c1.mul_(0.75)                                                   # what a replay restores is the layer as it is then
    want, want_scale = dl.dequant_fp4()
    for _ in range(2):
        q.zero_(), s.zero_(), v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(q, want) and same(s, want_scale) and same(v, b.vptq_fp4_values(want, want_scale, 1100))


def test_results_behind_work_that_is_still_running(b):
    """Every call directly behind the kernel that makes its operands, and in front of one that overwrites them."""
    g = gen(8)
    base = torch.randn(512, 2048, generator=g, device="cuda")
    x, wv = torch.empty(64, 2048, dtype=torch.float16, device="cuda"), torch.empty(512, 2048, device="cuda")
    for i in range(20):
        torch.mul(base, 1.0 + i, out=wv)
        x.copy_(base[:64] * (1 + i))
        w, s = b.vptq_fp4_quantize(wv)
        y = b.vptq_linear_fp4(x, w, s, out_dtype="fp32")
        z = b.vptq_linear_fp4(x[:3], w, s, out_dtype="fp32")
        x.zero_(), wv.zero_()
        w2, s2 = w.clone(), s.clone()
        w.zero_(), s.zero_()
        torch.cuda.synchronize()
        x.copy_(base[:64] * (1 + i))
        assert same(y, b.vptq_linear_fp4(x, w2, s2, out_dtype="fp32")) and same(z, b.vptq_linear_fp4(x[:3].clone(), w2, s2, out_dtype="fp32"))


# ---- waits that run out: every result is right or a NaN, and the next call is right ----------------------------

@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("B", [1, 16, 300])
def test_products_right_behind_their_weight(b, B, graph):
    """A weight that the kernel just before makes, of a size whose loads begin ahead of the tokens' quantization; another one every time."""
    M, N = 28672, 2080
    g = gen(B)
    x = torch.randn(B, N, generator=g, device="cuda").bfloat16()
    weights = [torch.randn(M, N, generator=g, device="cuda").bfloat16() for _ in range(3)]
    want = []
    for v in weights:
        w, s = b.vptq_fp4_quantize(v)
        torch.cuda.synchronize()
        want.append(b.vptq_linear_fp4(x, w, s))
        torch.cuda.synchronize()
    given, q = weights[0].clone(), torch.empty(M, N, device="cuda", dtype=torch.bfloat16)

    def both():
        q.copy_(given)
        return b.vptq_linear_fp4(x, *b.vptq_fp4_quantize(q))

    if graph:
        both()
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            y = both()
    got = []
    for i in range(9):
        given.copy_(weights[i % 3])
        if graph:
            captured.replay()
            got.append(y.clone())
        else:
            got.append(both())
    assert all(same(r, want[i % 3]) for i, r in enumerate(got))


@pytest.mark.parametrize("x_type", ["bf16", "e2m1"])
@pytest.mark.parametrize("M,N,B", [(37888, 320, 100), (9472, 4096, 100), (4096, 2048, 300), (8192, 8192, 2048), (4741, 416, 133), (128, 8192, 40), (1000, 4096, 77),
                                   (2048, 2048, 128), (28672, 8192, 16), (28672, 8192, 1), (4096, 16384, 7), (4096, 14336, 300), (1000, 16384, 500)])
def test_waits_that_run_out(b, M, N, B, x_type):
    g = gen(M + B)
    w, s = ref.random_weight(M, N, g, "cuda")
    x, xs = torch.randn(B, N, generator=g, device="cuda").bfloat16(), None
    if x_type == "e2m1":
        x, xs = b.vptq_fp4_quantize(x)
    room = torch.zeros(b.vptq_linear_fp4_workspace_bytes(b.make_fp4_desc(M, N, x_type, "fp32"), B), dtype=torch.uint8, device="cuda")
    call = lambda: b.vptq_linear_fp4(x, w, s, x_scale=xs, out_dtype="fp32", workspace=room)  # noqa: E731
    clean = call()
    assert b.vptq_workspace_status(room) == b.OK and torch.isfinite(clean).all()
    for _ in range(2):
        y = with_short_waits(b, call)
        assert b.vptq_workspace_status(room) == b.E_TIMEOUT
        right_or_nan(y, clean)
        assert same(call(), clean) and b.vptq_workspace_status(room) == b.OK


@pytest.mark.parametrize("clocks", [1, 200, 1000])
@pytest.mark.parametrize("M,N,B", [(4096, 4096, 1), (4736, 4096, 8), (300, 3990, 3)])
def test_waits_of_a_few_tokens_that_run_out(b, M, N, B, clocks):
    g = gen(M + B)
    cold = [ref.random_weight(M, N, g, "cuda") for _ in range(20)]     # (more than L2 holds)
    x = torch.randn(B, N, generator=g, device="cuda").half()
    clean = [b.vptq_linear_fp4(x, w, s, out_dtype="fp32") for w, s in cold]
    ys = with_short_waits(b, lambda: [b.vptq_linear_fp4(x, w, s, out_dtype="fp32") for w, s in cold], clocks)
    for y, want, (w, s) in zip(ys, clean, cold):
        right_or_nan(y, want, some=False)
        assert torch.isfinite(want).all() and same(b.vptq_linear_fp4(x, w, s, out_dtype="fp32"), want)


@pytest.mark.parametrize("clocks", [200, 800, 1600, 3200, 6400, 12800])
def test_waits_that_run_out_midway(b, clocks):
    g = gen(5)
    w, s = ref.random_weight(8192, 8192, g, "cuda")
    x = torch.randn(600, 8192, generator=g, device="cuda").half()
    room = torch.zeros(1 << 23, dtype=torch.uint8, device="cuda")
    for B in (1, 8, 16, 40, 100, 130, 300, 600):
        call = lambda: b.vptq_linear_fp4(x[:B], w, s, out_dtype="fp32", workspace=room)  # noqa: E731, B023
        clean = call()
        for _ in range(3):
            y = with_short_waits(b, call, clocks)
            right_or_nan(y, clean, some=False)
            assert b.vptq_workspace_status(room) == b.E_TIMEOUT or same(y, clean)
            assert same(call(), clean)
