"""Sparse tensors of the device are refused by every entry point that takes tensors; they have neither the memory nor the strides that these ask for."""
import pytest
import torch

from paper_2409_17066_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def test_sparse_tensors(b):
    x = torch.eye(64, device="cuda", dtype=torch.float16)
    w, s = b.vptq_fp4_quantize(x)
    w8, s8 = b.vptq_fp8_quantize(x, 128)
    cache = b.make_cache(2, 4, 2, 64)
    k = torch.ones(3, 2, 64, device="cuda")
    table, start, cu = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([[0, 1]], [0], [0, 3]))
    dl = b.DeviceLayer(synth.make_layer(synth.LayerSpec("q", 64, 64, v=8, k1=16), 0, 3, 1))
    thin = lambda t: t.to_sparse()  # noqa: E731
    calls = [lambda: b.vptq_fp4_quantize(thin(x)), lambda: b.vptq_fp8_quantize(thin(x), 128), lambda: b.vptq_fp4_values(thin(w), s, 64), lambda: b.vptq_fp4_values(w, thin(s), 64),
             lambda: b.vptq_fp4_values(w, s, 64, out=thin(x)), lambda: b.vptq_linear_fp4(thin(x), w, s), lambda: b.vptq_linear_fp4(x, thin(w), s), lambda: b.vptq_linear_fp4(x, w, thin(s)),
             lambda: b.vptq_linear_fp4(x, w, s, out=thin(x)), lambda: b.vptq_linear_fp4(x, w, s, workspace=thin(x)), lambda: b.vptq_linear_fp8(thin(x), w8, s8),
             lambda: b.vptq_linear_fp8(x, w8, s8, workspace=thin(x)), lambda: b.vptq_cache_write(thin(k), k, *cache, table, start, cu), lambda: b.vptq_cache_write(k, thin(k), *cache, table, start, cu),
             lambda: b.vptq_cache_write(k, k, *cache, thin(table), start, cu), lambda: b.vptq_cache_write(k, k, *cache, table, start, thin(cu)),
             lambda: b.vptq_cache_read(*cache[:3], thin(cache[3]), table, start, cu, 3, 64), lambda: b.vptq_cache_read(*cache, table, start, cu, 3, 64, "fp32", k=thin(k)),
             lambda: b.vptq_dequant_fp4(dl.desc, dl.ptrs, workspace=thin(x)), lambda: b.vptq_dequant_fp8(dl.desc, dl.ptrs, workspace=thin(x))]
    for call in calls:
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: dl.linear(thin(x)), lambda: b.vptq_dequant(dl.desc, dl.ptrs, thin(x))):
        with pytest.raises((AssertionError, RuntimeError)):
            call()
    # ... and what is not sparse is still taken
    assert torch.equal(b.vptq_fp4_values(w, s, 64, "fp16"), x)
