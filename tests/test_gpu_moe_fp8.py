"""The mixture-of-experts layer for a few tokens against its definition in 64 bits."""
import pytest
import torch

import fp8_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def layer(hidden, inner, experts, T, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, hidden, generator=g, device="cuda").to(TYPES[dtype])
    router = (torch.randn(experts, hidden, generator=g, device="cuda") * 0.05).to(TYPES[dtype])
    return x, router, *ref.random_experts(experts, inner, hidden, g, "cuda"), *ref.random_experts(experts, inner, hidden, g, "cuda"), \
        *ref.random_experts(experts, hidden, inner, g, "cuda")


def close(y, want):
    """h is rounded to e4m3 from sums that differ in their last FP32 bits: about 2^-20 of a value away, it falls on the other side of a
    tie, one in every 2^-3 of the value, for some 2^-16 of the values, which are then off by 2^-3 each: 2^-8 * 2^-3 of the whole by root mean
    square.  Twice that, and the result's own rounding."""
    off = float((y.double() - want).norm() / want.norm())
    assert off < 2.0 ** -10 + torch.finfo(y.dtype).eps / 2, off


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("hidden,inner,experts,top,T", [(256, 128, 4, 2, 1), (16, 16, 1, 1, 1), (128, 100, 8, 3, 2), (333, 200, 5, 5, 3), (1000, 333, 7, 2, 8),
                                                        (2048, 256, 64, 8, 1), (512, 144, 256, 16, 5), (264, 1030, 3, 1, 9), (640, 512, 6, 2, 16),
                                                        (2400, 272, 8, 4, 32), (4800, 1024, 4, 2, 4), (136, 2100, 12, 6, 31)])
def test_moe(b, hidden, inner, experts, top, T, renormalize, dtype):
    args = layer(hidden, inner, experts, T, dtype, hidden + T)
    out = torch.full((T, hidden), float("nan"), device="cuda")
    y = b.vptq_moe_fp8(*args, top, renormalize, out=out)
    assert y is out
    close(y, ref.moe(*args, top, renormalize))
    assert torch.equal(y, b.vptq_moe_fp8(*args, top, renormalize, out=torch.empty_like(out)))             # the same bits again
    z = b.vptq_moe_fp8(*args, top, renormalize)
    assert z.dtype == args[0].dtype and torch.equal(z, y.to(z.dtype))                                      # one rounding of the same sums


def test_more_than_eight_tokens_of_one_expert(b):
    args = layer(384, 272, 6, 29, "fp16", 3)
    x, router = args[0], args[1]
    x.abs_()
    router.zero_()
    router[4] = 1.0                                   # everyone's first choice; the rest are equal: experts 0 and 1 come next
    close(b.vptq_moe_fp8(*args, 3, out=torch.empty(29, 384, device="cuda")), ref.moe(*args, 3, True))


def test_equal_logits_go_to_the_lowest_expert(b):
    args = layer(256, 160, 40, 3, "bf16", 4)
    args[1][:] = args[1][0].clone()
    want = ref.moe(*args, 5, False)
    close(b.vptq_moe_fp8(*args, 5, False, out=torch.empty(3, 256, device="cuda")), want)
    for w in args[2::2]:                              # what the others hold does not matter
        w[5:].view(torch.uint8).fill_(0x7F)
    close(b.vptq_moe_fp8(*args, 5, False, out=torch.empty(3, 256, device="cuda")), want)


def test_extreme_logits(b):
    args = layer(128, 128, 8, 2, "bf16", 5)
    args[0][0] = 1.0
    args[1].mul_(2000)                                # the softmax is all one expert's: the others' weights are zeros
    close(b.vptq_moe_fp8(*args, 4, out=torch.empty(2, 128, device="cuda")), ref.moe(*args, 4, True))


def test_not_a_number_stays_in_its_token(b):
    args = layer(512, 256, 8, 6, "fp16", 6)
    clean = b.vptq_moe_fp8(*args, 2)
    args[0][2, 7] = float("nan")
    args[0][4, 300] = float("inf")
    y = b.vptq_moe_fp8(*args, 2)
    assert torch.isnan(y[2]).all() and torch.isnan(y[4]).all()
    # (the others share their experts with tokens 2 and 4 or not: their own sums are the same)
    for t in (0, 1, 3, 5):
        assert torch.equal(y[t], clean[t])


def test_writes_its_result_and_nothing_else(b):
    T, hidden = 5, 264
    args = layer(hidden, 128, 6, T, "fp16", 7)
    room = torch.full(((T + 2) * hidden,), 77.0, dtype=torch.float16, device="cuda")
    out = room[hidden:-hidden].view(T, hidden)
    desc = b.make_moe_desc(hidden, 128, 6, 2, "fp16", "fp16")
    ws = torch.full((b.vptq_moe_fp8_workspace_bytes(desc, T) + 256,), 255, dtype=torch.uint8, device="cuda")       # what it held does not matter
    b.vptq_moe_fp8(*args, 2, out=out, workspace=ws[:-256])
    assert (room[:hidden] == 77).all() and (room[-hidden:] == 77).all() and (ws[-256:] == 255).all()
    assert torch.equal(out, b.vptq_moe_fp8(*args, 2))


def test_streams_and_replayed_graphs(b):
    args = layer(1024, 512, 16, 4, "bf16", 8)
    want = b.vptq_moe_fp8(*args, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = b.vptq_moe_fp8(*args, 4)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first = b.vptq_moe_fp8(*args, 4)
        second = b.vptq_moe_fp8(first, *args[1:], 4)              # two layers, one after the other
    args[0].mul_(0.7)
    one = b.vptq_moe_fp8(*args, 4)
    two = b.vptq_moe_fp8(one, *args[1:], 4)
    for _ in range(3):
        first.zero_(), second.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, one) and torch.equal(second, two)


def test_the_most_tokens_experts_and_choices(b):
    args = layer(136, 48, 256, 32, "bf16", 10)
    close(b.vptq_moe_fp8(*args, 16, out=torch.empty(32, 136, device="cuda")), ref.moe(*args, 16, True))


@pytest.mark.parametrize("T", [1, 8, 32])
def test_two_calls_at_once(b, T):
    args = layer(1024, 512, 32, T, "bf16", 11)
    other = (args[0] * 0.5, *args[1:])
    want, want_other = b.vptq_moe_fp8(*args, 4), b.vptq_moe_fp8(*other, 4)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i, a in enumerate((args, other)):
            with torch.cuda.stream(streams[i]):
                got[i].append(b.vptq_moe_fp8(*a, 4))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got[0]) and all(torch.equal(y, want_other) for y in got[1])


def test_experts_and_router_written_just_before(b):
    layers = [layer(512, 384, 8, 3, "fp16", 20 + i) for i in range(4)]
    want = []
    for a in layers:
        want.append(b.vptq_moe_fp8(*a, 2))
        torch.cuda.synchronize()
    room = [torch.empty_like(t) for t in layers[0]]
    for a, w in zip(layers, want):
        for to, t in zip(room, a):
            to.view(torch.uint8).copy_(t.view(torch.uint8))
        assert torch.equal(b.vptq_moe_fp8(*room, 2), w)


def test_a_layers_experts_made_by_the_quantizer(b):
    """The operators together: experts quantized block by block when they are loaded, the layer for single tokens, and the same experts'
    projections through vptq_linear_fp8 for a prompt."""
    g = torch.Generator(device="cuda").manual_seed(9)
    hidden, inner, experts = 256, 384, 4
    def expert_weights(rows, cols):
        both = [b.vptq_fp8_quantize((torch.randn(rows, cols, generator=g, device="cuda") * 0.05).half(), 128) for _ in range(experts)]
        return torch.stack([q.view(torch.uint8) for q, _ in both]).view(torch.float8_e4m3fn), torch.stack([s for _, s in both])
    gate, up, down = expert_weights(inner, hidden), expert_weights(inner, hidden), expert_weights(hidden, inner)
    router = torch.zeros(experts, hidden, device="cuda", dtype=torch.float16)
    router[2] = 1
    x = torch.rand(20, hidden, generator=g, device="cuda").half()
    y = torch.cat([b.vptq_moe_fp8(x[i:i + 1], router, *gate, *up, *down, 1, out=torch.empty(1, hidden, device="cuda")) for i in range(20)])
    prompt = [b.vptq_linear_fp8(x, w[0][2], w[1][2], out_dtype="fp32") for w in (gate, up)]
    h = prompt[0] / (1 + torch.exp(-prompt[0])) * prompt[1]
    q, s = b.vptq_fp8_quantize(h)
    close(b.vptq_linear_fp8(q, down[0][2], down[1][2], x_scale=s, out_dtype="fp32"), y.double())
