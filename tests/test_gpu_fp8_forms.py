"""The forms that the kernels of the 8-bit floating point operators take for large layers, each against its definition in 64 bits."""
import pytest
import torch

import fp8_reference as ref
from paper_2409_17066_b200 import synth
from test_gpu_fp8 import check_linear, check_quantized, same
from test_gpu_moe_fp8 import close, layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


# ---- few tokens over many rows: passes of up to five groups of 16 rows -----------------------------------------

@pytest.mark.parametrize("x_type", ["e4m3", "fp16", "bf16"])
@pytest.mark.parametrize("M,N,B,passes", [(4800, 400, 1, 1),           # three groups a CTA, for some two: boxes of both heights
                                          (4737, 1024, 8, 1),          # the fewest rows, the last group with one of them
                                          (11840, 256, 3, 1),          # five groups, 80 rows: a pass lies in two 128-row blocks
                                          (12000, 333, 5, 2),          # passes of three and of two
                                          (18990, 640, 2, 2),          # of five and four, four and four
                                          (18990, 2320, 7, 2),         # more blocks of columns than a warp's ring has stages
                                          (26000, 130, 8, 3)])
def test_linear_few_tokens_many_rows(b, M, N, B, passes, x_type):
    if x_type == "e4m3":
        N = ref.pitch(N)
    groups = -(-M // 16)
    assert groups > 2 * sms()                                          # the kernel's rule for this form
    if sms() == 148:
        most = -(-groups // 148)                                       # of a CTA
        assert -(-most // 5) == passes
    check_linear(b, M, N, B, x_type, "fp32")


# ---- few tokens, long rows: stages of several blocks of columns --------------------------------------------------

@pytest.mark.parametrize("x_type", ["e4m3", "fp16", "bf16"])
@pytest.mark.parametrize("M,N,B", [(2400, 4096, 1),                    # two groups a CTA, for some one; two blocks a stage
                                   (4096, 4096 + 128, 8),              # 33 blocks: the last run is short
                                   (1000, 4096, 3), (17, 8192, 5),     # one group: four blocks a stage from 8192 columns on
                                   (2368, 8192 + 3 * 128, 2),          # 67 blocks: three of four in the last run
                                   (2380, 16384 - 128, 8)])
def test_linear_few_tokens_long_rows(b, M, N, B, x_type):
    check_linear(b, M, N, B, x_type, "fp32")


@pytest.mark.parametrize("M,N,B", [(15, 100, 8), (17, 129, 8), (130, 1030, 8), (260, 333, 8), (384, 2048, 8)])
@pytest.mark.parametrize("x_type", ["e4m3", "fp16", "bf16"])
def test_linear_eight_tokens(b, M, N, B, x_type):
    check_linear(b, M, ref.pitch(N) if x_type == "e4m3" else N, B, x_type, "fp32")


# ---- experts: down projections of two blocks of columns a stage -----------------------------------------------------

@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("hidden,inner,experts,top,T", [(512, 1024, 8, 4, 3), (640, 2176, 4, 2, 8),          # 17 blocks: a run is short
                                                        (4800, 2048, 4, 2, 16),                              # two groups of rows a pass, two passes
                                                        (2384, 1152, 6, 4, 32), (256, 4096, 3, 1, 9), (2048, 1024, 64, 8, 1)])
def test_moe_down_projection_in_runs(b, hidden, inner, experts, top, T, dtype):
    assert inner % 128 == 0 and inner // 128 * top >= 32               # the kernel's rule for two blocks a stage
    args = layer(hidden, inner, experts, T, dtype, hidden + T)
    y = b.vptq_moe_fp8(*args, top, out=torch.empty(T, hidden, device="cuda"))
    close(y, ref.moe(*args, top, True))
    assert same(y, b.vptq_moe_fp8(*args, top, out=torch.empty(T, hidden, device="cuda")))


# ---- restores with both tables in shared memory ----------------------------------------------------------------------

STAGED = [synth.LayerSpec("f_s8_256_256", 1203, 1301, v=8, k1=256, k2=256), synth.LayerSpec("f_s8_4096_256", 6000, 2064, v=8, k1=4096, k2=256),
          synth.LayerSpec("f_s8_256_4096", 6001, 2062, v=8, k1=256, k2=4096, n_out=7, v0=8, k0=256),
          synth.LayerSpec("f_s6_4096_256_out", 4300, 2206, v=6, k1=4096, k2=256, n_out=33, v0=4, k0=64),
          synth.LayerSpec("f_s6_256_256", 1100, 1300, v=6, k1=256, k2=256)]


@pytest.mark.parametrize("spec", STAGED, ids=lambda s: s.name)
def test_dequant_fp8_with_main_and_residual_table_staged(b, spec):
    # the kernel's rule: more table reads a CTA, two of them an SM, than there are entries, which fit beside the block
    assert spec.R * spec.Nc // (2 * sms()) > spec.k1 + spec.k2 <= 4992
    dl = b.DeviceLayer(synth.make_layer(spec, 0, 3, 1))
    check_quantized(*dl.dequant_fp8(), dl.dequant(), 128)
