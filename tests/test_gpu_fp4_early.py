"""Products whose weight loads begin ahead of the call's own quantization of the tokens (large weights; the more tokens, the smaller), directly behind the
kernel that makes the weight: another one every time, and the results of a call that waits for all of it."""
import pytest
import torch

from test_gpu_fp4 import gen, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("M,N,tokens", [(28672, 5888, (1, 16, 95)), (12100, 4192, (95, 96, 300, 700))])
def test_right_behind_the_weight(b, M, N, tokens, graph):
    g = gen(M)
    weights = [b.vptq_fp4_quantize(torch.randn(M, N, generator=g, device="cuda").bfloat16()) for _ in range(3)]
    q, s = (t.clone() for t in weights[0])
    scales = [w[1] for w in weights]
    values = [b.vptq_fp4_values(*w, N) for w in weights]             # (quantized again they are the same codes and scales)
    given = values[0].clone()
    for B in tokens:
        x = torch.randn(B, N, generator=g, device="cuda").bfloat16()
        torch.cuda.synchronize()
        want = [b.vptq_linear_fp4(x, *w, out_dtype="fp32") for w in weights]
        torch.cuda.synchronize()

        def both():
            w, ws = b.vptq_fp4_quantize(given)
            return b.vptq_linear_fp4(x, w, ws, out_dtype="fp32"), w, ws  # noqa: B023

        if graph:
            both()
            torch.cuda.synchronize()
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                y, w, ws = both()
        for i in range(6):
            given.copy_(values[i % 3])
            if graph:
                captured.replay()
                got = y.clone()
            else:
                got, w, ws = both()
            assert same(ws, scales[i % 3]) and same(got, want[i % 3]), (B, i)
            # ... and a weight overwritten in place by a copy, in front of the call and behind it
            q.copy_(weights[(i + 1) % 3][0]), s.copy_(scales[(i + 1) % 3])
            got = b.vptq_linear_fp4(x, q, s, out_dtype="fp32")
            q.zero_(), s.zero_()
            assert same(got, want[(i + 1) % 3]), (B, i)
