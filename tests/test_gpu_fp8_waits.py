"""Device-side waits of the 8-bit floating point kernels that run out: every result is right or a NaN, and the next call is right."""
import pytest
import torch

import fp8_reference as ref
from test_gpu_fp8 import same
from test_gpu_moe_fp8 import layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def with_short_waits(b, call, clocks=1):
    """call() while waits are abandoned after so many clocks: with 1, the first that is not satisfied already."""
    torch.cuda.synchronize()
    try:
        b.lib.vptq_debug_set_wait_limit(clocks)
        y = call()
        torch.cuda.synchronize()
    finally:
        b.lib.vptq_debug_set_wait_limit(0)
    return y


def right_or_nan(y, clean, some=True):
    lost = torch.isnan(y)
    assert ((y == clean) | lost).all() and (lost.any() or not some), float(lost.float().mean())


# (235 MB: far more than is on its way when a warp looks for its first blocks.  Rows of FP16 values that are no multiple of 16 bytes are read
# one value at a time, for longer than the weights take: no wait need run out there.)
@pytest.mark.parametrize("x_type", ["fp16", "e4m3"])
@pytest.mark.parametrize("M,N,B", [(28672, 8192, 1), (28000, 8190, 8), (4736, 49152, 3)])
def test_few_tokens(b, M, N, B, x_type):
    g = torch.Generator(device="cuda").manual_seed(M + B)
    w, s = ref.random_weight(M, N, g, "cuda")
    x, xs = torch.randn(B, N, generator=g, device="cuda").half(), None
    if x_type == "e4m3":
        x, xs = b.vptq_fp8_quantize(x)
    call = lambda: b.vptq_linear_fp8(x, w, s, x_scale=xs, out_dtype="fp32")  # noqa: E731
    clean = call()
    assert torch.isfinite(clean).all()
    for _ in range(2):
        right_or_nan(with_short_waits(b, call), clean, some=x_type == "e4m3" or N % 8 == 0)
        assert same(call(), clean)


@pytest.mark.parametrize("hidden,inner,experts,top,T", [(2048, 8192, 8, 2, 8), (2048, 1024, 64, 8, 1), (4096, 3000, 6, 3, 29), (1000, 4000, 12, 6, 4)])
def test_experts(b, hidden, inner, experts, top, T):
    args = layer(hidden, inner, experts, T, "bf16", hidden + T)
    call = lambda: b.vptq_moe_fp8(*args, top, out=torch.empty(T, hidden, device="cuda"))  # noqa: E731
    clean = call()
    assert torch.isfinite(clean).all()
    for _ in range(2):
        right_or_nan(with_short_waits(b, call), clean)
        assert same(call(), clean)


# (tiles of one CTA, of a pair, and tiles split over the 2, 4 and 8 CTAs of a cluster; results that go out by copies and by stores)
@pytest.mark.parametrize("x_type", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,N,B", [(37888, 160, 100), (9472, 4096, 100), (4096, 2048, 300), (8192, 8192, 2048), (4741, 208, 133), (128, 4096, 40), (1000, 2048, 77),
                                   (2048, 1024, 128), (28672, 8192, 16)])
def test_many_tokens(b, M, N, B, x_type):
    g = torch.Generator(device="cuda").manual_seed(M + B)
    w, s = ref.random_weight(M, N, g, "cuda")
    x, xs = torch.randn(B, N, generator=g, device="cuda").bfloat16(), None
    if x_type == "e4m3":
        x, xs = b.vptq_fp8_quantize(x)
    room = torch.zeros(b.vptq_linear_fp8_workspace_bytes(b.make_fp8_desc(M, N, x_type, "fp32"), B), dtype=torch.uint8, device="cuda")
    call = lambda: b.vptq_linear_fp8(x, w, s, x_scale=xs, out_dtype="fp32", workspace=room)  # noqa: E731
    clean = call()
    assert b.vptq_workspace_status(room) == b.OK and torch.isfinite(clean).all()
    for _ in range(2):
        y = with_short_waits(b, call)
        assert b.vptq_workspace_status(room) == b.E_TIMEOUT
        right_or_nan(y, clean)
        assert same(call(), clean) and b.vptq_workspace_status(room) == b.OK


@pytest.mark.parametrize("clocks", [200, 800, 1600, 3200, 6400, 12800])
def test_waits_that_run_out_midway(b, clocks):
    """Some waits of a call run out and others do not: nothing that depends on a lost one may look right."""
    g = torch.Generator(device="cuda").manual_seed(5)
    w, s = ref.random_weight(8192, 8192, g, "cuda")
    x = torch.randn(600, 8192, generator=g, device="cuda").half()
    args = layer(2048, 8192, 8, 8, "bf16", 3)
    room = torch.zeros(1 << 23, dtype=torch.uint8, device="cuda")
    calls = [lambda: b.vptq_moe_fp8(*args, 2, out=torch.empty(8, 2048, device="cuda"))]
    calls += [lambda B=B: b.vptq_linear_fp8(x[:B], w, s, out_dtype="fp32", workspace=room) for B in (1, 8, 40, 100, 300, 600)]
    for i, call in enumerate(calls):
        clean = call()
        for _ in range(3):
            y = with_short_waits(b, call, clocks)
            right_or_nan(y, clean, some=False)
            if i > 2:
                assert b.vptq_workspace_status(room) == b.E_TIMEOUT or same(y, clean)
            assert same(call(), clean)
