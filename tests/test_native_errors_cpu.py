"""What torch throws inside the native entry points reaches Python as an error; it does not end the process.  (The calls are made by a child process, one
after the other: one that does end it fails its own test and those behind it.)"""
import subprocess
import sys

import pytest

CALLS = {  # call -> error
    "b.vptq_fp4_quantize(sparse)": "AssertionError",
    "b.vptq_fp8_quantize(sparse)": "AssertionError",
    "b.vptq_fp4_values(sparse.byte(), sparse.byte(), 32)": "AssertionError",
    "b.vptq_linear_fp4(sparse, sparse, sparse)": "AssertionError",
    "b.vptq_linear_fp8(sparse, sparse, sparse)": "AssertionError",
    "b.vptq_cache_write(*[sparse] * 9)": "AssertionError",
    "b.vptq_cache_read(*[sparse] * 7, 3, 64)": "AssertionError",
    "b.vptq_dequant_fp4(d, p, workspace=dense)": "AssertionError",
    "b.vptq_dequant_fp4(d, p, workspace=sparse)": "AssertionError",
    "b.vptq_dequant_fp8(d, p, workspace=sparse)": "AssertionError",
    "b._native.linear(d, dense, p, dense, sparse)": "RuntimeError",
}
CHILD = """
import sys, torch
from paper_2409_17066_b200 import binding as b
sparse, dense = torch.eye(3).to_sparse(), torch.eye(3)
d, p = b.make_desc(64, 64, 8, 256, 0, flags=0), b.LayerPtrs(0x1000, 0x1000)
for call in sys.argv[1:]:
    try:
        eval(call)
    except Exception as e:
        print(call, "->", type(e).__name__, flush=True)
"""


@pytest.fixture(scope="module")
def answers():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    r = subprocess.run([sys.executable, "-c", CHILD, *CALLS], capture_output=True, text=True, timeout=300)
    return r.stdout.splitlines()


@pytest.mark.parametrize("call", CALLS)
def test_sparse_tensors(answers, call):
    assert f"{call} -> {CALLS[call]}" in answers
