"""Calls of the 8-bit floating point operators that a program makes beside the plain ones: slices of stacked operands, empty batches,
workspaces and layers in other memory, logits that are zeros of both signs,
restores in a graph."""
import pytest
import torch

import fp8_reference as ref
from paper_2409_17066_b200 import synth
from test_gpu_fp8 import same
from test_gpu_moe_fp8 import layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


# ---- scales that start at any multiple of four bytes ---------------------------------------------------

@pytest.mark.parametrize("B", [3, 40])
def test_every_expert_of_a_stack_takes_a_prompt(b, B):
    g = torch.Generator(device="cuda").manual_seed(1)
    w, s = ref.random_experts(4, 256, 384, g, "cuda")                  # 2 x 3 scales an expert: 24 bytes from one to the next
    x = torch.randn(B, 384, generator=g, device="cuda").half()
    for e in range(4):
        assert s[e].data_ptr() % 16 == 8 * (e % 2)
        assert same(b.vptq_linear_fp8(x, w[e], s[e]), b.vptq_linear_fp8(x, w[e], s[e].clone()))


@pytest.mark.parametrize("B", [3, 40])
def test_some_tokens_of_a_quantized_batch(b, B):
    g = torch.Generator(device="cuda").manual_seed(2)
    w, s = ref.random_weight(130, 384, g, "cuda")
    q, qs = b.vptq_fp8_quantize(torch.randn(B + 3, 384, generator=g, device="cuda"))
    for t in range(1, 4):
        assert qs[t:].data_ptr() % 16 != 0
        got = b.vptq_linear_fp8(q[t:t + B], w, s, x_scale=qs[t:t + B], out_dtype="fp32")
        want = b.vptq_linear_fp8(q[t:t + B].clone(), w, s, x_scale=qs[t:t + B].clone(), out_dtype="fp32")
        assert same(got, want)


def test_layers_of_a_stack_of_experts(b):
    one, two = (layer(256, 384, 3, 2, "bf16", 30 + i) for i in range(2))
    both = [torch.stack([p.view(torch.uint8), q.view(torch.uint8)]).view(p.dtype) if p.dtype == torch.float8_e4m3fn else torch.stack([p, q])
            for p, q in zip(one, two)]
    assert any(t[1].data_ptr() % 16 for t in both[3::2])
    for i, a in enumerate((one, two)):
        assert same(b.vptq_moe_fp8(*[t[i] for t in both], 2), b.vptq_moe_fp8(*a, 2))


def test_slices_of_scales_in_a_replayed_graph(b):
    g = torch.Generator(device="cuda").manual_seed(3)
    w, s = ref.random_experts(2, 256, 384, g, "cuda")
    x = torch.randn(20, 384, generator=g, device="cuda").half()
    b.vptq_linear_fp8(x, w[1], s[1].clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = b.vptq_linear_fp8(x, w[1], s[1])
    s.mul_(1.5)                                                        # what a replay reads is what the scales hold then
    want = b.vptq_linear_fp8(x, w[1], s[1].clone())
    for _ in range(2):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(y, want)


# ---- empty batches ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("x_type", ["fp16", "bf16", "e4m3"])
def test_an_empty_batch_through_the_operators(b, x_type):
    g = torch.Generator(device="cuda").manual_seed(4)
    w, s = ref.random_weight(130, 256, g, "cuda")
    x, xs = torch.empty(0, 256, device="cuda", dtype=torch.bfloat16 if x_type == "bf16" else torch.float16), None
    if x_type == "e4m3":
        x, xs = b.vptq_fp8_quantize(x)
    y = b.vptq_linear_fp8(x, w, s, x_scale=xs)
    assert tuple(y.shape) == (0, 130) and y.dtype == (torch.float16 if x_type == "fp16" else torch.bfloat16)
    out = torch.empty(0, 130, device="cuda")
    assert b.vptq_linear_fp8(x, w, s, x_scale=xs, out=out) is out
    with pytest.raises(AssertionError):
        b.vptq_linear_fp8(x, w, s, x_scale=xs, out=torch.empty(0, 131, device="cuda"))
    with pytest.raises(b.VptqError):                                   # what else is refused still is
        b.vptq_linear_fp8(torch.empty(0, 256, device="cuda"), w, s)


def test_an_empty_batch_through_the_experts(b):
    args = layer(256, 128, 4, 2, "fp16", 5)
    y = b.vptq_moe_fp8(args[0][:0], *args[1:], 2)
    assert tuple(y.shape) == (0, 256) and y.dtype == torch.float16
    out = torch.empty(0, 256, device="cuda")
    assert b.vptq_moe_fp8(args[0][:0], *args[1:], 2, out=out) is out
    with pytest.raises(b.VptqError):
        b.vptq_moe_fp8(args[0][:0], *args[1:], 5)


# ---- a workspace that the kernels cannot write ---------------------------------------------------------------

def test_a_workspace_elsewhere_is_refused(b):
    g = torch.Generator(device="cuda").manual_seed(7)
    w, s = ref.random_weight(130, 256, g, "cuda")
    x = torch.randn(20, 256, generator=g, device="cuda").half()
    args = layer(256, 128, 4, 2, "fp16", 8)
    spread = torch.zeros(1 << 21, 2, dtype=torch.uint8, device="cuda")[:, 0]              # every other byte: not all of it is the workspace's
    for room in (torch.zeros(1 << 22, dtype=torch.uint8), spread):
        with pytest.raises(AssertionError, match="workspace"):
            b.vptq_linear_fp8(x, w, s, workspace=room)
        with pytest.raises(AssertionError, match="workspace"):
            b.vptq_moe_fp8(*args, 2, workspace=room)
    assert not spread.any()


def test_a_layer_in_host_memory_is_refused(b):
    desc = b.make_desc(64, 64, 8, 256)
    streams = [torch.zeros(1 << 14, dtype=torch.uint8) for _ in range(4)]
    idx, table, scale, bias = (t.data_ptr() for t in streams)
    with pytest.raises(AssertionError, match="current device"):
        b.vptq_dequant_fp8(desc, b.LayerPtrs(idx, table, None, None, None, None, scale, bias))
    streams = [t.cuda() for t in streams]                              # the same layer where it belongs: zeros, with one scale
    q, s = b.vptq_dequant_fp8(desc, b.LayerPtrs(streams[0].data_ptr(), streams[1].data_ptr(), None, None, None, None, streams[2].data_ptr(), streams[3].data_ptr()))
    assert q.device == s.device == streams[0].device and not q.view(torch.uint8).any()


# ---- zeros of both signs are equal logits -------------------------------------------------------------------

def test_logits_that_vanish_go_to_the_lowest_experts(b):
    # products of 1e-60 are zeros in FP32, below zero for the first experts and above for the others: all logits are equal
    args = layer(1024, 128, 40, 1, "bf16", 6)
    args[0].fill_(1e-30)
    args[3].mul_(1e30), args[5].mul_(1e30)                             # (the experts' results are ordinary values all the same)
    args[1].fill_(1e-30)
    args[1][:7] = -1e-30
    got = b.vptq_moe_fp8(*args, 3, False, out=torch.empty(1, 1024, device="cuda"))
    args[1].zero_()
    want = b.vptq_moe_fp8(*args, 3, False, out=torch.empty(1, 1024, device="cuda"))
    assert want.any() and same(got, want)


# ---- restores in a graph -------------------------------------------------------------------------------------

@pytest.mark.parametrize("permuted", [False, True])
def test_a_restore_in_a_replayed_graph(b, permuted):
    spec = synth.LayerSpec("f_graph", 1000, 1100, v=8, k1=256, k2=16, permuted=permuted)
    dl = b.DeviceLayer(synth.make_layer(spec, 0, 3, 1))
    dl.dequant_fp8()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, s = dl.dequant_fp8()
    dl.c1.mul_(0.75)                                                   # what a replay restores is the layer as it is then
    want, want_scale = dl.dequant_fp8()
    for _ in range(2):
        q.view(torch.uint8).zero_(), s.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(q, want) and same(s, want_scale)
